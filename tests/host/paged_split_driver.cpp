// The paged attention's plan with its real split rule, under sanitizers: over
// random calls every new row is some own job's, every key is in its splits, the
// parts stay inside the workspace, and the kernels' dispatch has the waves and
// tiles that a job asks for. Only the launches are stand-ins; they record the
// jobs.
#include <stdarg.h>
#include <stdio.h>
#include <stdlib.h>

#include <algorithm>
#include <random>
#include <vector>

#include "../../include/zsa.h"
#include "../../paper_2509_01190_amd/csrc/zsa_internal.h"

namespace {
struct Job {
  zsa::PagedAttention a;
  bool many;
};
long g_checks = 0;
int g_cus = 256, g_joined = 0, g_dtype = -1, g_launches = 0, g_round = 0;
std::vector<Job> g_jobs;

void expect(bool ok, const char* what) {
  ++g_checks;
  if (!ok) {
    fprintf(stderr, "call %d: %s (%s)\n", g_round, what, zsa_last_error());
    exit(1);
  }
}
}  // namespace

extern "C" const char* hipGetErrorString(hipError_t) { return "hip stub"; }

namespace zsa {
static char g_text[512];
int set_error(int code, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_text, sizeof(g_text), fmt, ap);
  va_end(ap);
  return code;
}
int device_cu_count() { return g_cus; }
hipError_t launch_paged_append(hipStream_t, int, const PagedAppend&) { return hipSuccess; }
hipError_t launch_paged_attention(hipStream_t, int dtype, const PagedAttention* few, int fews, const PagedAttention* many, int manys) {
  ++g_launches;
  g_dtype = dtype;
  for (int i = 0; i < fews; ++i) g_jobs.push_back({few[i], false});
  for (int i = 0; i < manys; ++i) g_jobs.push_back({many[i], true});
  return hipSuccess;
}
hipError_t launch_paged_join(hipStream_t, int, const float2*, const float*, int parts, int, int, int, void*, int64_t, float*) {
  g_joined = parts;
  return hipSuccess;
}
}  // namespace zsa
extern "C" const char* zsa_last_error(void) { return zsa::g_text; }

// what the kernels of one launch take for granted
static void check_launch(int hd) {
  const bool matrix = zsa::paged_matrix(g_dtype, hd);
  const int width = hd * (g_dtype == ZSA_BF16 ? 2 : 4);
  int fews = 0, manys = 0, waves = 0, tile = 0, head = -1;
  for (const Job& j : g_jobs) {
    expect(j.a.hd == hd && (head < 0 || j.a.head_len == head), "one head width, one prefix before the rows");
    head = j.a.head_len;
    if (j.many) {
      ++manys;
      expect(matrix && j.a.tile == zsa::kPagedManyRows, "many rows: the bf16 matrix kernels'");
    } else {
      expect(fews++ == 0 || (j.a.waves == waves && j.a.tile == tile), "one width of workgroups a launch");
      waves = j.a.waves;
      tile = j.a.tile;
    }
    expect(j.a.splits >= 1 && j.a.chunk >= 128 && j.a.chunk % 128 == 0, "splits");
    expect(static_cast<int64_t>(j.a.splits) * j.a.chunk < INT32_MAX, "keys in 32 bits");
    expect(zsa::paged_blocks(j.a, j.many) * (waves == 8 || (j.many && hd == 128) ? 512 : 256) < (int64_t{1} << 32), "a grid");
    const int64_t pairs = static_cast<int64_t>(j.a.splits) * (j.a.H / j.a.G) * j.a.B;
    for (int64_t pair = std::max<int64_t>(pairs - 8, 0); pair < pairs; ++pair)  // the kernels' places of the last tiles
      expect((j.many ? ((pair >> 3) * j.a.tiles + j.a.tiles - 1) * 8 + (pair & 7) : pair + pairs * (j.a.tiles - 1)) <
                 zsa::paged_blocks(j.a, j.many), "a workgroup for every tile");
  }
  expect(fews <= 2 && manys <= 2, "two jobs of a kind");
  if (fews == 0) return;
  expect(waves == 4 || (manys == 0 && tile == zsa::kPagedFewRows && (waves == 1 || (waves == 8 && (matrix || width <= 256)))),
         "waves that the dispatch has");
  expect(tile == zsa::kPagedFewRows || (!matrix && tile == 32), "rows that the dispatch has");
}

int main() {
  void* A = reinterpret_cast<void*>(0x100000);
  const int32_t* I = reinterpret_cast<const int32_t*>(0x200000);
  std::mt19937 g(7);
  auto pick = [&](int64_t n) { return static_cast<int64_t>(g() % static_cast<uint32_t>(n)); };
  // up to `most`, spread over the orders of magnitude
  auto far = [&](int64_t most) { return pick((most >> pick(30)) + 1); };
  const int cus[6] = {256, 256, 256, 304, 32, 1};
  int refused = 0, waves[9] = {}, manys = 0, heads = 0, prefixes = 0;
  for (g_round = 0; g_round < 30000; ++g_round) {
    zsa_paged_kv kv{};
    const int hds[4] = {16, 32, 64, 128};
    g_cus = cus[pick(6)];
    kv.head_dim = hds[pick(4)];
    kv.n_kv_heads = 1 + pick(pick(2) ? 4 : 40);
    const int G = 1 + pick(9), H = kv.n_kv_heads * G;
    kv.dtype = pick(2);
    kv.page_size = 16 << pick(6);
    const int64_t longest = 1 << 30;
    kv.max_pages = static_cast<int32_t>(far(longest / kv.page_size));
    kv.table_stride = kv.max_pages;
    kv.n_pages = 1 + pick(1000);
    kv.page_stride = 2LL * kv.n_kv_heads * kv.head_dim * kv.page_size;
    kv.pool = A;
    kv.table = I;
    const int batch = 1 + pick(pick(4) ? 20 : 300), kind = pick(3);
    std::vector<int32_t> cu(batch + 1, 0);
    for (int b = 0; b < batch; ++b) cu[b + 1] = cu[b] + (kind == 0 ? 1 : kind == 1 ? pick(40) : pick(8) ? 1 : pick(2000));
    const int T = cu[batch];
    const int max_len = static_cast<int>(std::min<int64_t>(far(longest), static_cast<int64_t>(kv.max_pages) * kv.page_size));
    const int prefix = pick(2) ? static_cast<int>(far(longest)) : 0;
    if (T == 0) continue;
    const size_t need = zsa_paged_attention_workspace_size(&kv, H, batch, cu.data(), max_len, prefix);
    const int64_t width = static_cast<int64_t>(H) * kv.head_dim, rows = static_cast<int64_t>(T) * H;
    g_jobs.clear();
    g_joined = g_launches = 0;
    const int rc = zsa_prefix_attention(nullptr, &kv, A, width, H, 1, 0.1f, batch, cu.data(), I, I, max_len, I, prefix, A, width,
                                        nullptr, need > 0 ? A : nullptr, need);
    if (rc == ZSA_EUNSUPPORTED) {  // more workgroups than a grid holds
      expect(g_launches == 0, "refused before its launch");
      ++refused;
      continue;
    }
    expect(rc == ZSA_OK && g_launches == 1 && g_dtype == kv.dtype, "a launch");
    check_launch(kv.head_dim);
    bool common = false, direct = false;
    for (const Job& j : g_jobs) {
      const zsa::PagedAttention& a = j.a;
      const bool prefixes_own = a.cu == nullptr;
      const int64_t len = prefixes_own ? prefix : (a.head_len + 31) / 32 * 32 + static_cast<int64_t>(max_len);
      expect(static_cast<int64_t>(a.chunk) * a.splits >= len, "every key is in a split");
      expect(a.max_len == (prefixes_own ? prefix : max_len), "the keys' number");
      if (prefixes_own) expect(static_cast<int64_t>(a.tile) * a.tiles >= static_cast<int64_t>(T) * G, "the prefix's rows");
      common |= (prefixes_own || a.head_len > 0) && prefix > 0;
      direct |= a.direct != 0;
      expect(!a.direct || (a.splits == 1 && (g_joined == 0 || a.ml != nullptr)), "rows finished at once");
      if (a.ml != nullptr) {
        const int64_t part = a.ml - static_cast<float2*>(A);
        expect(part % rows == 0 && a.splits <= a.parts, "parts inside the joined ones");
        // (a row's parts are all written: those that its job has not, as empty ones)
        expect(prefixes_own ? part == 0 && a.parts == a.splits : part / rows + a.parts == g_joined, "every part is written");
        expect(reinterpret_cast<char*>(a.o + a.parts * rows * kv.head_dim) <= static_cast<char*>(A) + need, "inside the workspace");
        expect(reinterpret_cast<char*>(a.ml + a.parts * rows) <= reinterpret_cast<char*>(a.o), "maxima before sums");
      } else {
        expect(a.direct && g_joined == 0 && need == 0, "finished rows");
      }
      if (!j.many) ++waves[a.waves];
      manys += j.many;
      heads += a.head_len > 0;
      prefixes += prefixes_own;
    }
    expect(common == (prefix > 0) && !(direct && prefix > 0 && g_jobs[0].a.cu == nullptr), "the prefix is some job's");
    // every sequence with new rows is one own job's, which has a tile for each of them
    for (int b = 0; b < batch; ++b) {
      const int64_t n = static_cast<int64_t>(cu[b + 1] - cu[b]) * G;
      int own = 0;
      for (const Job& j : g_jobs) {
        if (j.a.cu == nullptr || (j.many ? n <= j.a.few_rows : n > j.a.few_rows)) continue;
        ++own;
        expect(static_cast<int64_t>(j.a.tile) * j.a.tiles >= n, "tiles for all rows");
      }
      expect(n == 0 || own == 1, "one job for a sequence's rows");
    }
  }
  expect(waves[1] > 100 && waves[4] > 100 && waves[8] > 100 && manys > 100 && heads > 100 && prefixes > 100, "all plans were met");
  expect(refused < 30000 / 4, "most calls go through");
  printf("ok %ld refused %d waves %d %d %d many %d heads %d prefixes %d\n", g_checks, refused, waves[1], waves[4], waves[8], manys,
         heads, prefixes);
  return 0;
}
