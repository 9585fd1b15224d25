// C entry points of the paged key/value cache: argument checks, the split of
// the keys over workgroups and the workspace for the parts. As in
// zsa_api.cpp, everything only enqueues work on the caller's stream.
#include <algorithm>
#include <math.h>

#include "../../include/zsa.h"
#include "zsa_check.h"
#include "zsa_internal.h"

namespace {

using zsa::check_dtype;
using zsa::check_head_dim;
using zsa::check_kv_heads;
using zsa::check_ptr16;
using zsa::check_seqs;
using zsa::check_width;
using zsa::esize;
using zsa::round256;
using zsa::set_error;

#define CHECK(expr)                \
  do {                             \
    const int rc_ = (expr);        \
    if (rc_ != ZSA_OK) return rc_; \
  } while (0)

#define HIP_TRY(expr, what)                                                                    \
  do {                                                                                         \
    const hipError_t e_ = (expr);                                                              \
    if (e_ != hipSuccess) return set_error(ZSA_EHIP, "%s: %s", what, hipGetErrorString(e_)); \
  } while (0)

// the cache's description; `rows`: the call has rows that use the table
int check_cache(const zsa_paged_kv* c, bool rows) {
  if (c == nullptr) return set_error(ZSA_EINVAL, "kv is NULL");
  CHECK(check_dtype(c->dtype));
  CHECK(check_head_dim(c->head_dim));
  if (c->n_kv_heads <= 0) return set_error(ZSA_EINVAL, "n_kv_heads %d", c->n_kv_heads);
  if (c->page_size < 16 || c->page_size > (1 << 20) || (c->page_size & (c->page_size - 1)) != 0)
    return set_error(ZSA_EUNSUPPORTED, "page_size %d (a power of two from 16 to 2^20)", c->page_size);
  if (c->n_pages < 0 || c->max_pages < 0)
    return set_error(ZSA_ESHAPE, "n_pages %d, max_pages %d", c->n_pages, c->max_pages);
  CHECK(check_ptr16(c->pool, "pool", !rows || c->n_pages == 0));
  if (rows && c->table == nullptr && c->max_pages > 0) return set_error(ZSA_EINVAL, "table is NULL");
  if (c->table_stride < c->max_pages)
    return set_error(ZSA_ESHAPE, "table_stride %lld < max_pages %d", (long long)c->table_stride, c->max_pages);
  CHECK(check_width(c->dtype, c->page_stride, "page_stride"));
  const int64_t row = 2 * static_cast<int64_t>(c->n_kv_heads) * c->head_dim;
  if (row > (1 << 20)) return set_error(ZSA_EUNSUPPORTED, "%d key/value heads of %d", c->n_kv_heads, c->head_dim);
  if (c->page_stride < row * c->page_size)
    return set_error(ZSA_ESHAPE, "page_stride %lld shorter than a page of %d rows of %lld",
                     (long long)c->page_stride, c->page_size, (long long)row);
  // the kernels reach a page's rows through 32-bit byte offsets
  if (row * c->page_size * static_cast<int64_t>(esize(c->dtype)) >= (int64_t{1} << 31))
    return set_error(ZSA_EUNSUPPORTED, "pages of 2 GiB or more");
  return ZSA_OK;
}

zsa::PagedRows rows_of(const zsa_paged_kv& c) {
  zsa::PagedRows r{};
  r.pool = c.pool;
  r.page_stride = c.page_stride;
  r.shift = __builtin_ctz(static_cast<unsigned>(c.page_size));
  r.n_pages = c.n_pages;
  r.table = c.table;
  r.table_stride = c.table_stride;
  r.max_pages = c.max_pages;
  r.kvd = c.n_kv_heads * c.head_dim;
  return r;
}

int check_stride(int32_t dtype, int64_t stride, int64_t width, const char* name) {
  CHECK(check_width(dtype, stride, name));
  if (stride < width) return set_error(ZSA_ESHAPE, "%s %lld < %lld columns", name, (long long)stride, (long long)width);
  return ZSA_OK;
}

size_t parts_bytes(int64_t parts, int64_t rows, int hd) {
  return round256(parts * rows * sizeof(float2)) + round256(parts * rows * hd * sizeof(float));
}

// Packed rows (new rows times query heads per key/value head) up to which a
// sequence goes to the few-row kernel: one or two workgroups of 16, where the
// rows are read twice. us, two / the many-row kernel, 8 sequences, 32 packed
// rows, 32 heads of 128 on 8: up to 508 rows 10.0 / 15.5, up to 3008 31.2 / 23.7;
// 17 to 32 rows, 32 heads of 64, up to 2032 36.6 / 33.3. A common prefix, with
// other parts to join in any case, of 4000 rows, 32 heads of 64: 40 rows 22.6 /
// 26.3, 63 rows 30.5 / 33.4, of 6000, 32 of 128 on 8, 48 rows 17.0 / 16.5. More rows
// of a prefix where what the workgroups of 16 read, mostly from the L2s, is at
// most 192 MB, in smaller heads 64 MB, and they are at most two a CU (32 of 128
// on 8: 240 rows on 3000 22.9 / 25.6, on 8000 47 / 31; 12 of 64: 240 on 800 15.3 /
// 18.7; 24 of 64 on 8: 180 on 3000, 74 MB, 18.8 / 18.1). Where
// all workgroups of 16 rows run at once (`fits`), up to eight of them over up to
// 1536 rows: 34 sequences of up to 756 rows, 8 to 72 packed rows, 8 heads of 128
// on 1, 12.1 / 19.3; 3 of 60 to 100 rows over up to 600, 12 of 64, 8.4 / 19.0; 12 of
// 20 new rows over up to 1320, 24 of 64 on 8, 17.4 / 21.9; with more than run at
// once it loses (25 of 10 to 20 rows over up to 920, 32 of 128 on 8, 35.1 / 24.7).
// Two over up to 3040 in heads below 128 and at most one a CU (`one`): 12 of 8 new
// rows, 24 of 64 on 8, 18.6 / 22.5; 40, with more, 68 / 59; 12, 32 of 128 on 8, 37.4
// / 34.7.
int few_rows(int max_len, int hd, bool fits, bool one) {
  if (fits && max_len <= 1536) return 128;
  return max_len <= (one && hd < 128 ? 3040 : 1024) ? 32 : 16;
}
bool few_prefix(int hd, int kv_heads, int64_t rows, int prefix) {
  const int64_t workgroups = (rows + 15) / 16 * kv_heads;
  return rows <= (hd < 128 ? 64 : 32) || (workgroups <= 2 * zsa::device_cu_count() &&
                                          workgroups * hd * 4.0 * prefix <= (hd < 128 ? 64 : 192) * 1048576.0);
}

// The rows of one kind: the common prefix's, or the own ones of the sequences
// of few packed rows, or of many.
struct Part {
  bool many;
  int tile, tiles;    // packed rows of a workgroup; of the longest sequence, how many of those
  int waves;          // of a few-row workgroup
  int chunk, splits;  // 0 splits: there are none
  bool head;          // the common prefix goes before the sequences' rows, in the same workgroups
};

// The parts of the prefix come first, the others' after them, in the same places.
struct Plan {
  Part prefix, few, many;
  int few_rows;  // packed rows up to which a sequence is one of the few
  int own() const { return std::max(few.splits, many.splits); }
  int parts() const { return prefix.splits + own(); }
  // rows are finished at once where they have no other part
  bool direct(const Part& l) const { return prefix.splits == 0 && l.splits == 1; }
  bool join() const { return parts() > 1; }
};

Plan plan_of(const zsa_paged_kv& kv, int H, int batch, const int32_t* cu, int max_len, int prefix) {
  Plan p{};
  const int hd = kv.head_dim;
  const int64_t G = H / kv.n_kv_heads, T = cu[batch];
  const bool matrix = zsa::paged_matrix(kv.dtype, hd);
  int64_t longest = 0, sixteens = 0;  // packed rows of a sequence; blocks of 16 of all
  for (int b = 0; b < batch; ++b) {
    const int64_t rows = (cu[b + 1] - cu[b]) * G;
    longest = std::max(longest, rows);
    sixteens += (rows + 15) / 16;
  }
  const int64_t row = 2 * static_cast<int64_t>(kv.n_kv_heads) * hd * esize(kv.dtype);
  // (what LDS holds of the few-row kernels' workgroups, a CU)
  const int resident = 512 / (hd * static_cast<int>(esize(kv.dtype)));
  const bool fits = sixteens * kv.n_kv_heads <= static_cast<int64_t>(zsa::device_cu_count()) * std::min(resident, 4);
  // A short prefix goes before the sequences' rows, in the same workgroups:
  //  * those of few rows read it once per sequence, from the L2s, where that is at
  //    most 32 MB, or with the own rows 160 and no parts are to join then (8
  //    sequences of up to 41 rows behind 501, 12 heads of 64: 15.0 -> 10.7 us; 30 x 4
  //    rows over up to 100 behind 700, 32 of 128 on 8, 98 MB, 22.1 -> 12.6, 60 over
  //    up to 1000 behind 500, 370 MB, 36.9 -> 44.6; fp32, 55 x 4 over 10 behind 99,
  //    49 MB, 40 -> 25.7);
  //  * those of many rows take no part's bytes and no join for it, but are more
  //    than the rows of all together would be (`more` us): 5 of up to 757 rows
  //    behind 226, 8 heads of 128 on 1, 77.6 -> 36.3; 8 of up to 200 behind 1000, 32
  //    of 128 on 8, 56.0 -> 42.2, behind 3000 95.2 -> 91.4; 1 of 300 behind 300, 12 of
  //    64, 17.2 -> 18.5.
  const bool head = prefix > 0 && max_len < (1 << 29) && prefix < (1 << 29);
  const int whole = head ? (prefix + 31) / 32 * 32 + max_len : 0;
  int limit;
  int64_t most[2];
  auto sort = [&](int len) {
    limit = p.few_rows = few_rows(len, hd, fits && longest <= 128, sixteens * kv.n_kv_heads <= zsa::device_cu_count());
    most[0] = most[1] = 0;
    for (int b = 0; b < batch; ++b) {
      const int64_t rows = (cu[b + 1] - cu[b]) * G;
      const bool many = matrix && rows > limit;
      most[many] = std::max(most[many], rows);
    }
  };
  double other = 0;  // us of the few-row work: its cached rows, half the longest each, at 5 TB/s
  const int max_own = max_len;
  // (`beside` as in paged_chunk)
  auto part = [&](bool many, int64_t max_rows, int max_len, bool common, int beside) {
    Part l{};
    l.many = many;
    // fp32: 32 rows a workgroup cost less than twice 16, and more than 16 on
    // another CU. One launch takes one width: the sequences' own, and 32 where the
    // prefix is nearly all the work and long (in 16s / 32s, us: 60 rows behind 4000,
    // 32 heads of 128 on 8, own rows up to 500, 94 / 111; 55 behind 300 24.7 / 30.4;
    // 120 behind 12000, 16 heads of 64 on 2, 99 / 77).
    const double pairs = static_cast<double>(T) * G * prefix;
    const bool wide = common ? p.few.tile == 32 || (pairs * kv.n_kv_heads * hd >= 7e8 && pairs >= 64.0 * batch * max_own)
                             : !fits;
    l.tile = many ? zsa::kPagedManyRows : !matrix && max_rows > 16 && wide ? 32 : zsa::kPagedFewRows;
    l.tiles = static_cast<int>((max_rows + l.tile - 1) / l.tile);
    int64_t workgroups = common ? l.tiles : 0, packed = common ? T * G : 0;
    for (int b = 0; b < batch && !common; ++b) {
      const int64_t rows = (cu[b + 1] - cu[b]) * G;
      if (many != (matrix && rows > limit)) continue;
      workgroups += (rows + l.tile - 1) / l.tile;
      packed += rows;
    }
    l.waves = beside == 0 && !many ? zsa::paged_waves(matrix, kv.dtype, hd, l.tile, max_len, workgroups * kv.n_kv_heads) : 4;
    l.chunk = zsa::paged_chunk(many, matrix, hd, max_len, workgroups * kv.n_kv_heads, packed * kv.n_kv_heads,
                               !common && batch > 1, beside, other, &l.splits);
    if (!many) other += workgroups * kv.n_kv_heads * hd * 2.0 * esize(kv.dtype) * max_len / 2 / 5e6;
    return l;
  };
  if (head) {
    sort(whole);
    int64_t fews = 0, tiles = 0, many_rows = 0;
    for (int b = 0; b < batch; ++b) {
      const int64_t rows = (cu[b + 1] - cu[b]) * G;
      const bool many = matrix && rows > limit;
      fews += !many && rows > 0;
      if (!many) continue;
      tiles += (rows + zsa::kPagedManyRows - 1) / zsa::kPagedManyRows;
      many_rows += rows;
    }
    const double again = static_cast<double>(fews) * prefix * row / (1 << 20);
    const double own = again / prefix * max_len;
    const int64_t common = (T * G + zsa::kPagedManyRows - 1) / zsa::kPagedManyRows;
    const double more = static_cast<double>(std::max<int64_t>(tiles - common, 0)) * kv.n_kv_heads * prefix / 64 * 1.5 / zsa::device_cu_count();
    const double parts = 4 + 2.0 * many_rows * kv.n_kv_heads * hd * 8 / 2e6;
    if ((again <= 32 || again + own <= 160) && (tiles == 0 || more <= parts)) {
      p.few = p.many = Part{};
      if (most[0] > 0) p.few = part(false, most[0], whole, false, most[1] > 0);
      if (most[1] > 0) p.many = part(true, most[1], whole, false, 0);
      p.few.head = p.many.head = true;
      if (again <= 32 || p.own() == 1) return p;
      p.few = p.many = Part{};
      other = 0;
    }
  }
  sort(max_len);
  if (most[0] > 0) p.few = part(false, most[0], max_len, false, prefix > 0 ? 2 : most[1] > 0);
  if (most[1] > 0) p.many = part(true, most[1], max_len, false, prefix > 0 ? 2 : 0);
  if (prefix > 0) {
    // (one launch takes one width of tiles)
    p.prefix = part(matrix && !few_prefix(hd, kv.n_kv_heads, T * G, prefix), T * G, prefix, true, 2);
    if (!matrix && p.few.splits > 0 && p.few.tile != p.prefix.tile) {
      p.few.tile = p.prefix.tile;
      p.few.tiles = static_cast<int>((most[0] + p.few.tile - 1) / p.few.tile);
    }
  }
  return p;
}

size_t workspace_of(const Plan& p, const zsa_paged_kv& kv, int T, int H) {
  return p.join() ? parts_bytes(p.parts(), static_cast<int64_t>(T) * H, kv.head_dim) : 0;
}

int attention(void* stream, const zsa_paged_kv* kv, const void* q, int64_t q_stride, int32_t n_heads,
              int32_t causal, float scale, int32_t batch, const int32_t* cu_host, const int32_t* cu_dev,
              const int32_t* kv_len, int32_t max_kv_len, const int32_t* prefix_pages, int32_t prefix_len,
              void* out, int64_t out_stride, float* lse, void* ws, size_t ws_bytes) {
  int32_t T, max_new;
  CHECK(check_seqs(batch, cu_host, cu_dev, &T, &max_new));
  CHECK(check_cache(kv, T > 0));
  int G = 1;
  if (n_heads <= 0) return set_error(ZSA_EINVAL, "n_heads %d", n_heads);
  CHECK(check_kv_heads(n_heads, kv->n_kv_heads, &G));
  if (!(scale > 0.f)) return set_error(ZSA_EINVAL, "scale must be positive");
  if (max_kv_len < 0 || prefix_len < 0)
    return set_error(ZSA_EINVAL, "max_kv_len %d, prefix_len %d", max_kv_len, prefix_len);
  const int64_t width = static_cast<int64_t>(n_heads) * kv->head_dim;
  CHECK(check_stride(kv->dtype, q_stride, width, "q_stride"));
  CHECK(check_stride(kv->dtype, out_stride, width, "out_stride"));
  CHECK(check_ptr16(q, "q", T == 0));
  CHECK(check_ptr16(out, "out", T == 0));
  if (T > 0 && kv_len == nullptr) return set_error(ZSA_EINVAL, "kv_len is NULL");
  if (T > 0 && prefix_len > 0 && prefix_pages == nullptr) return set_error(ZSA_EINVAL, "prefix_pages is NULL");
  if (max_kv_len > static_cast<int64_t>(kv->max_pages) * kv->page_size)
    return set_error(ZSA_ESHAPE, "max_kv_len %d beyond the table's %d pages of %d rows", max_kv_len, kv->max_pages,
                     kv->page_size);
  if (max_kv_len > (1 << 30) || prefix_len > (1 << 30))
    return set_error(ZSA_EUNSUPPORTED, "max_kv_len %d, prefix_len %d beyond 2^30", max_kv_len, prefix_len);
  if (static_cast<int64_t>(T) * n_heads >= (int64_t{1} << 30))
    return set_error(ZSA_EUNSUPPORTED, "%d rows of %d heads: 2^30 or more", T, n_heads);
  if (T == 0) return ZSA_OK;
  const Plan p = plan_of(*kv, n_heads, batch, cu_host, max_kv_len, prefix_len);
  const size_t need = workspace_of(p, *kv, T, n_heads);
  if (ws_bytes < need) return set_error(ZSA_EWORKSPACE, "workspace %zu bytes < %zu", ws_bytes, need);
  if (need > 0) CHECK(check_ptr16(ws, "ws"));
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int64_t rows = static_cast<int64_t>(T) * n_heads;
  float2* ml = p.join() ? static_cast<float2*>(ws) : nullptr;
  float* o = p.join() ? reinterpret_cast<float*>(static_cast<char*>(ws) + round256(p.parts() * rows * sizeof(float2))) : nullptr;
  zsa::PagedAttention a{};
  a.at = rows_of(*kv);
  a.q = q;
  a.q_stride = q_stride;
  a.cu = cu_dev;
  a.kv_len = kv_len;
  a.max_len = max_kv_len;
  a.T = T;
  a.B = batch;
  a.H = n_heads;
  a.G = G;
  a.hd = kv->head_dim;
  a.causal = causal != 0;
  a.scale = scale;
  a.out = out;
  a.out_stride = out_stride;
  a.lse = lse;
  // The call's cached rows, half the longest each. From 64 MB on, a quarter of
  // the last-level cache, a program with more than one layer finds none of them
  // there again.
  const double cached = (batch * 0.5 * max_kv_len + prefix_len) * 2 * kv->n_kv_heads * kv->head_dim * esize(kv->dtype);
  // the work of the few-row kernel and of the many-row one
  zsa::PagedAttention job[2][2];
  int jobs[2] = {0, 0};
  int64_t threads = 0;
  for (const Part* l : {&p.prefix, &p.few, &p.many}) {
    if (l->splits == 0) continue;
    zsa::PagedAttention& x = job[l->many][jobs[l->many]++];
    x = a;
    const bool prefix = l == &p.prefix;
    x.tile = l->tile;
    x.tiles = l->tiles;
    x.waves = l->waves;
    x.once = cached >= 64e6;
    x.chunk = l->chunk;
    x.splits = l->splits;
    x.few_rows = prefix ? (l->many ? 0 : INT32_MAX) : p.many.splits > 0 ? p.few_rows : INT32_MAX;
    x.parts = prefix ? l->splits : p.own();
    x.direct = p.direct(*l);
    if (l->head) {
      x.head_table = prefix_pages;
      x.head_len = prefix_len;
    }
    if (prefix) {
      x.at.table = prefix_pages;
      x.at.max_pages = static_cast<int>((static_cast<int64_t>(prefix_len) + kv->page_size - 1) / kv->page_size);
      x.cu = nullptr;
      x.kv_len = nullptr;
      x.max_len = prefix_len;
      x.B = 1;
      x.causal = 0;
      x.direct = 0;
    }
    if (ml != nullptr) {
      x.ml = ml + (prefix ? 0 : p.prefix.splits) * rows;
      x.o = o + (prefix ? 0 : p.prefix.splits) * rows * kv->head_dim;
    }
    threads += zsa::paged_blocks(x, l->many) * (l->waves == 8 || (l->many && kv->head_dim == 128) ? 512 : 256);
  }
  // (what a grid holds; the join takes head_dim / 4 threads a row, eight times that at most)
  if (std::max(threads, p.join() ? rows * kv->head_dim / 4 : 0) >= (int64_t{1} << 32) - 4096)
    return set_error(ZSA_EUNSUPPORTED, "%d sequences of up to %d rows of %d heads: more workgroups than a grid holds",
                     batch, max_new, n_heads);
  HIP_TRY(zsa::launch_paged_attention(s, kv->dtype, job[0], jobs[0], job[1], jobs[1]), "paged attention");
  if (p.join())
    HIP_TRY(zsa::launch_paged_join(s, kv->dtype, ml, o, p.parts(), T, n_heads, kv->head_dim, out, out_stride, lse),
            "paged attention's parts");
  return ZSA_OK;
}

}  // namespace

extern "C" {

int zsa_paged_append(void* stream, const zsa_paged_kv* kv, const void* k, int64_t k_stride, const void* v,
                     int64_t v_stride, const void* q, int64_t q_stride, int32_t n_heads, void* q_out,
                     int64_t q_out_stride, const int32_t* pos, float rope_theta, int32_t batch,
                     const int32_t* cu_host, const int32_t* cu_dev, const int32_t* kv_len) {
  int32_t T, max_new;
  CHECK(check_seqs(batch, cu_host, cu_dev, &T, &max_new));
  CHECK(check_cache(kv, T > 0));
  const int64_t kvd = static_cast<int64_t>(kv->n_kv_heads) * kv->head_dim;
  CHECK(check_ptr16(k, "k", T == 0));
  CHECK(check_ptr16(v, "v", T == 0));
  CHECK(check_stride(kv->dtype, k_stride, kvd, "k_stride"));
  CHECK(check_stride(kv->dtype, v_stride, kvd, "v_stride"));
  if (q != nullptr) {
    int G = 1;
    if (n_heads <= 0) return set_error(ZSA_EINVAL, "n_heads %d", n_heads);
    CHECK(check_kv_heads(n_heads, kv->n_kv_heads, &G));
    if (pos == nullptr) return set_error(ZSA_EINVAL, "q without pos: nothing would rotate it");
    CHECK(check_ptr16(q, "q"));
    CHECK(check_ptr16(q_out, "q_out"));
    const int64_t width = static_cast<int64_t>(n_heads) * kv->head_dim;
    CHECK(check_stride(kv->dtype, q_stride, width, "q_stride"));
    CHECK(check_stride(kv->dtype, q_out_stride, width, "q_out_stride"));
    if (q_out == q && q_out_stride != q_stride && T > 1)
      return set_error(ZSA_ESHAPE, "q_out is q with another stride: %lld, %lld", (long long)q_out_stride, (long long)q_stride);
  }
  if (pos != nullptr && !(rope_theta > 0.f)) return set_error(ZSA_EINVAL, "rope_theta <= 0");
  if (T > 0 && kv_len == nullptr) return set_error(ZSA_EINVAL, "kv_len is NULL");
  if (T >= (1 << 24)) return set_error(ZSA_EUNSUPPORTED, "%d rows in one call (2^24 or more)", T);
  if (T == 0) return ZSA_OK;
  zsa::PagedAppend a{};
  a.at = rows_of(*kv);
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.q_out = q_out;
  a.q_out_stride = q_out_stride;
  a.H = n_heads;
  a.Hkv = kv->n_kv_heads;
  a.hd = kv->head_dim;
  a.T = T;
  a.B = batch;
  a.pos = pos;
  a.cu = cu_dev;
  a.kv_len = kv_len;
  if (pos != nullptr) {
    // theta^(-2i/hd) by repeated products: off by 63 roundings at most, 7e-15
    // of an angle, which is 1e-9 rad at position 10^5; 64 powers take 2 us
    const double step = pow(static_cast<double>(rope_theta), -2.0 / kv->head_dim);
    a.inv_freq[0] = 1.0;
    for (int i = 1; i < kv->head_dim / 2; ++i) a.inv_freq[i] = a.inv_freq[i - 1] * step;
  }
  HIP_TRY(zsa::launch_paged_append(static_cast<hipStream_t>(stream), kv->dtype, a), "paged append");
  return ZSA_OK;
}

size_t zsa_paged_attention_workspace_size(const zsa_paged_kv* kv, int32_t n_heads, int32_t batch,
                                          const int32_t* cu_host, int32_t max_kv_len, int32_t prefix_len) {
  if (kv == nullptr || cu_host == nullptr || batch <= 0 || n_heads <= 0 || kv->n_kv_heads <= 0 ||
      n_heads % kv->n_kv_heads != 0 || max_kv_len < 0 || prefix_len < 0 || max_kv_len > (1 << 30) ||
      prefix_len > (1 << 30) || check_head_dim(kv->head_dim) != ZSA_OK || check_dtype(kv->dtype) != ZSA_OK)
    return 0;  // (the call itself refuses these)
  for (int b = 0; b < batch; ++b)
    if (cu_host[b + 1] < cu_host[b]) return 0;
  const int T = cu_host[batch];
  if (T <= 0) return 0;
  const Plan p = plan_of(*kv, n_heads, batch, cu_host, max_kv_len, prefix_len);
  return workspace_of(p, *kv, T, n_heads);
}

int zsa_paged_attention(void* stream, const zsa_paged_kv* kv, const void* q, int64_t q_stride, int32_t n_heads,
                        int32_t causal, float scale, int32_t batch, const int32_t* cu_host,
                        const int32_t* cu_dev, const int32_t* kv_len, int32_t max_kv_len, void* out,
                        int64_t out_stride, float* lse, void* ws, size_t ws_bytes) {
  return attention(stream, kv, q, q_stride, n_heads, causal, scale, batch, cu_host, cu_dev, kv_len, max_kv_len,
                   nullptr, 0, out, out_stride, lse, ws, ws_bytes);
}

int zsa_prefix_attention(void* stream, const zsa_paged_kv* kv, const void* q, int64_t q_stride, int32_t n_heads,
                         int32_t causal, float scale, int32_t batch, const int32_t* cu_host,
                         const int32_t* cu_dev, const int32_t* kv_len, int32_t max_kv_len,
                         const int32_t* prefix_pages, int32_t prefix_len, void* out, int64_t out_stride,
                         float* lse, void* ws, size_t ws_bytes) {
  return attention(stream, kv, q, q_stride, n_heads, causal, scale, batch, cu_host, cu_dev, kv_len, max_kv_len,
                   prefix_pages, prefix_len, out, out_stride, lse, ws, ws_bytes);
}

}  // extern "C"
