// Test shim: layers.cpp with a context made by hand and launchers that record
// what they were given, so that the host side of the layer calls (refusals,
// tilings, workspaces) runs without a GPU.
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <string>

#include "../paper_2606_11081_amd/csrc/layers.cpp"

namespace gasloc {
static std::string g_last;
std::string format(const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  std::vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return buf;
}
gasloc_status fail(gasloc_ctx* c, gasloc_status st, const std::string& msg) {
  g_last = msg;
  if (c) c->err = msg;
  return st;
}
gasloc_status hip_fail(gasloc_ctx* c, hipError_t, const char* what) { return fail(c, GASLOC_EDEVICE, what); }

int g_launches = 0;
static LinearArgs g_linear;
static EmbeddingGradArgs g_sums;
static NormGradArgs g_norm;
static int g_tile = 0, g_vec = 0, g_merges = 0;
hipError_t launch_embedding(const EmbeddingArgs&, int, int, hipStream_t) { return ++g_launches, hipSuccess; }
hipError_t launch_token_sort(const SortArgs&, hipStream_t) { return ++g_launches, hipSuccess; }
hipError_t launch_token_merge(const MergeArgs&, hipStream_t) { return ++g_merges, ++g_launches, hipSuccess; }
hipError_t launch_embedding_sums(const EmbeddingGradArgs& a, int, hipStream_t) {
  g_sums = a;
  return ++g_launches, hipSuccess;
}
hipError_t launch_embedding_join(const EmbeddingGradArgs&, hipStream_t) { return ++g_launches, hipSuccess; }
hipError_t launch_layer_norm(const NormArgs&, int, int, bool, hipStream_t) { return ++g_launches, hipSuccess; }
hipError_t launch_layer_norm_grad(const NormGradArgs& a, int, int, bool, hipStream_t) {
  g_norm = a;
  return ++g_launches, hipSuccess;
}
hipError_t launch_layer_norm_join(const NormGradArgs&, hipStream_t) { return ++g_launches, hipSuccess; }
int norm_waves(int width) { return width <= 2048 ? 1 : width <= 8192 ? 4 : 8; }
hipError_t launch_linear(const LinearArgs& a, LinearPass, int, int, int tile, bool vec, hipStream_t) {
  g_linear = a;
  g_tile = tile;
  g_vec = vec;
  return ++g_launches, hipSuccess;
}
}  // namespace gasloc

extern "C" {
gasloc_ctx* shim_context(int n, int64_t P, int dtype, int cus) {
  gasloc_ctx* c = new gasloc_ctx();
  c->n = n;
  c->P = P;
  c->hp.param_dtype = dtype;
  c->cus = cus;
  c->buf.x = reinterpret_cast<void*>(0x10000000);
  c->buf.y = reinterpret_cast<void*>(0x20000000);
  c->buf.ld = (P + 7) / 8 * 8;
  c->stepped.assign(static_cast<size_t>(n), 0);
  return c;
}
void shim_step(gasloc_ctx* c, int i) { c->stepped[static_cast<size_t>(i)] = 1; }
void shim_fail(gasloc_ctx* c) { c->failed = true; }
void shim_free(gasloc_ctx* c) { delete c; }
const char* shim_error() { return gasloc::g_last.c_str(); }
int shim_launches() { const int k = gasloc::g_launches; gasloc::g_launches = 0; return k; }
int shim_merges() { const int k = gasloc::g_merges; gasloc::g_merges = 0; return k; }
uint64_t shim_linear_stepped() { return gasloc::g_linear.w.stepped; }
// tile, vec, chunk, then n+1 tile starts, n+1 part starts, n workers
void shim_linear_plan(int n, int64_t* out) {
  *out++ = gasloc::g_tile;
  *out++ = gasloc::g_vec;
  *out++ = gasloc::g_linear.chunk;
  for (int i = 0; i <= n; ++i) *out++ = gasloc::g_linear.tiles.begin[i];
  for (int i = 0; i <= n; ++i) *out++ = gasloc::g_linear.parts.begin[i];
  for (int i = 0; i < n; ++i) *out++ = gasloc::g_linear.order[i];
}
// chunk, fill rows, then n+1 chunk starts
void shim_sums_plan(int n, int64_t* out) {
  *out++ = gasloc::g_sums.chunk;
  *out++ = gasloc::g_sums.fill_rows;
  for (int i = 0; i <= n; ++i) *out++ = gasloc::g_sums.chunks.begin[i];
}
// rows per tile, then n+1 tile starts
void shim_norm_plan(int n, int64_t* out) {
  *out++ = gasloc::g_norm.tile_rows;
  for (int i = 0; i <= n; ++i) *out++ = gasloc::g_norm.tiles.begin[i];
}
}
