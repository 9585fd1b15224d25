// Host code of the paged cache's entry points under sanitizers: refusals, the
// split of the work, and that what a call launches stays inside its
// workspace's parts. Device-side stand-ins record the jobs.
#include <stdarg.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <vector>

#include "../../include/zsa.h"
#include "../../paper_2509_01190_amd/csrc/zsa_internal.h"

namespace {
int g_checks = 0;
std::vector<zsa::PagedAttention> g_jobs;
int g_joined = 0, g_appends = 0;

void expect(bool ok, const char* what) {
  ++g_checks;
  if (!ok) {
    fprintf(stderr, "failed: %s (%s)\n", what, zsa_last_error());
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
int device_cu_count() { return 256; }
bool paged_matrix(int dtype, int hd) { return dtype == 1 && hd >= 32; }
int paged_waves(bool, int, int, int, int, int64_t) { return 4; }
int paged_chunk(bool many, bool, int, int max_len, int64_t workgroups, int64_t, bool, int, double, int* splits) {
  const int least = many ? 256 : 512, blocks = max_len > 0 ? (max_len + least - 1) / least : 1;
  const int want = workgroups > 64 ? 1 : blocks < 7 ? blocks : 7;
  const int per = (blocks + want - 1) / want;
  *splits = (blocks + per - 1) / per;
  return per * least;
}
int64_t paged_blocks(const PagedAttention& a, bool) {
  return static_cast<int64_t>(a.splits) * (a.H / a.G) * a.B * a.tiles;
}
hipError_t launch_paged_append(hipStream_t, int, const PagedAppend&) {
  ++g_appends;
  return hipSuccess;
}
hipError_t launch_paged_attention(hipStream_t, int, const PagedAttention* few, int fews, const PagedAttention* many, int manys) {
  g_jobs.insert(g_jobs.end(), few, few + fews);
  g_jobs.insert(g_jobs.end(), many, many + manys);
  return hipSuccess;
}
hipError_t launch_paged_join(hipStream_t, int, const float2*, const float*, int parts, int, int, int, void*, int64_t, float*) {
  g_joined = parts;
  return hipSuccess;
}
}  // namespace zsa
extern "C" const char* zsa_last_error(void) { return zsa::g_text; }

int main() {
  void* A = reinterpret_cast<void*>(0x100000);
  const int32_t* I = reinterpret_cast<const int32_t*>(0x200000);
  srand(3);
  for (int round = 0; round < 4000; ++round) {
    zsa_paged_kv kv{};
    const int hds[4] = {16, 32, 64, 128};
    kv.head_dim = hds[rand() % 4];
    kv.n_kv_heads = 1 + rand() % 12;
    const int G = 1 + rand() % 9, H = kv.n_kv_heads * G;
    kv.dtype = rand() % 2;
    kv.page_size = 16 << (rand() % 5);
    kv.max_pages = rand() % 300;
    kv.table_stride = kv.max_pages + rand() % 3;
    kv.n_pages = 1 + rand() % 1000;
    kv.page_stride = 2LL * kv.n_kv_heads * kv.head_dim * kv.page_size;
    kv.pool = A;
    kv.table = I;
    const int batch = rand() % 20;
    std::vector<int32_t> cu(batch + 1, 0);
    for (int b = 0; b < batch; ++b) cu[b + 1] = cu[b] + (rand() % 3 ? 1 : rand() % 200);
    const int T = cu[batch], max_len = kv.max_pages * kv.page_size ? rand() % (kv.max_pages * kv.page_size) : 0;
    const int prefix = rand() % 2 ? rand() % 5000 : 0;
    const size_t need = zsa_paged_attention_workspace_size(&kv, H, batch, cu.data(), max_len, prefix);
    const int64_t width = static_cast<int64_t>(H) * kv.head_dim;
    auto call = [&](void* ws, size_t n) {
      g_jobs.clear();
      g_joined = 0;
      return zsa_prefix_attention(nullptr, &kv, A, width, H, 1, 0.1f, batch, cu.data(), I, I, max_len, I, prefix, A,
                                  width, nullptr, ws, n);
    };
    if (T == 0) {
      expect(need == 0 && call(nullptr, 0) == ZSA_OK && g_jobs.empty(), "no rows");
      continue;
    }
    if (need > 0) {
      expect(call(A, need - 1) == ZSA_EWORKSPACE && g_jobs.empty(), "short workspace");
      expect(call(nullptr, need) == ZSA_EINVAL && g_jobs.empty(), "no workspace");
    }
    expect(call(need ? A : nullptr, need) == ZSA_OK, "attention");
    const int64_t rows = static_cast<int64_t>(T) * H;
    int covered = 0, own = 0;
    for (const zsa::PagedAttention& j : g_jobs) {
      expect(j.chunk % 128 == 0 && j.splits >= 1, "splits");
      const bool common = j.cu == nullptr;
      const int64_t len = common ? prefix : (j.head_len + 31) / 32 * 32 + max_len;
      expect(static_cast<int64_t>(j.chunk) * j.splits >= len, "the splits cover the keys");
      if (common || j.head_len == prefix) covered = prefix;
      own += !common;
      if (j.ml != nullptr) {
        const int64_t part = j.ml - static_cast<float2*>(A);
        expect(part % rows == 0 && part / rows + j.parts <= g_joined, "parts inside the joined ones");
        expect(reinterpret_cast<char*>(j.o + j.parts * rows * kv.head_dim) <= static_cast<char*>(A) + need, "inside the workspace");
        expect(reinterpret_cast<char*>(j.ml + j.parts * rows) <= reinterpret_cast<char*>(j.o), "maxima before sums");
      } else {
        expect(j.direct && g_joined == 0, "finished rows");
      }
    }
    expect(covered == prefix && own >= 1 && own <= 2, "every key is some job's");
    expect(zsa_paged_append(nullptr, &kv, A, width, A, width, nullptr, 0, 0, nullptr, 0, nullptr, 0.f, batch, cu.data(), I, I) ==
               (G >= 1 ? ZSA_OK : ZSA_ESHAPE), "append");
  }
  printf("ok %d\n", g_checks);
  return 0;
}
