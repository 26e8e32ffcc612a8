// C ABI of the layer operators (include/gasloc_layers.h): argument checks,
// tilings and workspace layouts of a call, kernel launches.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cmath>
#include <string>

#include "context.h"
#include "gasloc.h"
#include "gasloc_layers.h"
#include "internal.h"
#include "layers.h"

using gasloc::aligned16;
using gasloc::DeviceGuard;
using gasloc::fail;
using gasloc::format;
using gasloc::LiveRows;
using gasloc::param_bytes;
using gasloc::Spans;

namespace {

// A launch holds fewer than 2^32 threads.  Where there are many rows, at most 16 of them go with a row in the lookup,
// the sort, the merges, the sums and the norm's backward pass; the launches that may need more are checked: linear
// layers by kMaxGroups, the norm's forward pass and the zeroing of tables by check_launch.
constexpr int64_t kMaxRows = int64_t(1) << 27;
constexpr int64_t kMaxThreads = 0xffffffffll;
constexpr int64_t kMaxGroups = kMaxThreads / 512;  // of a linear layer's launch
constexpr int64_t kMaxLd = int64_t(1) << 21;

// Nothing but a status leaves the library: building a message may run out of memory.
template <typename F>
gasloc_status guarded(F&& body) {
  try {
    return body();
  } catch (...) {
    return GASLOC_ENOMEM;
  }
}

gasloc_status check_context(gasloc_ctx* c) {
  if (!c) return fail(nullptr, GASLOC_EINVAL, "NULL context");
  if (c->failed) return fail(c, GASLOC_ESTATE, "context unusable after a device error: " + c->err);
  return GASLOC_OK;
}

std::string check_rows(int n, const int64_t* row_ptr) {
  if (!row_ptr) return "row_ptr must not be NULL";
  if (row_ptr[0] != 0) return "row_ptr must start at 0";
  for (int i = 0; i < n; ++i)
    if (row_ptr[i + 1] < row_ptr[i]) return format("row_ptr decreases at worker %d", i);
  if (row_ptr[n] > kMaxRows) return "more than 2^27 rows";
  return "";
}

std::string check_types(const gasloc_ctx& c, int32_t dtype) {
  if (dtype != GASLOC_F32 && dtype != GASLOC_BF16) return "dtype must be F32 or BF16";
  if (dtype == GASLOC_F32 && c.hp.param_dtype != GASLOC_F32) return "F32 activations need F32 parameters";
  return "";
}

std::string check_columns(const gasloc_ctx& c, const char* what, int64_t begin, int64_t size) {
  if (begin < 0 || begin > c.P - size)
    return format("%s: columns [%lld, %lld) outside the worker's row of %lld", what, (long long)begin,
                  (long long)(begin + size), (long long)c.P);
  return "";
}

// An activation of `rows` rows of `cols` elements.
std::string check_act(const char* what, const void* p, int64_t ld, int64_t cols, int64_t rows, int32_t dtype) {
  if (rows > 0 && !p) return format("%s must not be NULL", what);
  if (reinterpret_cast<uintptr_t>(p) % param_bytes(dtype) != 0)
    return format("%s is not aligned to its elements", what);
  if (ld < cols || ld >= kMaxLd) return format("%s: row length must be in [%lld, 2^21)", what, (long long)cols);
  return "";
}

std::string check_launch(const char* what, int64_t groups, int64_t threads) {
  return groups * threads > kMaxThreads ? format("%s too large for one launch", what) : std::string();
}

// A result may take the place of an operand if their rows are the same.
std::string check_in_place(const char* what, const void* a, int64_t a_ld, const void* b, int64_t b_ld) {
  return a && a == b && a_ld != b_ld ? format("%s: rows of another length in the same place", what) : std::string();
}

std::string check_grads(const gasloc_ctx& c, const float* grads, int64_t grad_ld, int32_t accumulate) {
  if (!grads || !aligned16(grads)) return "grads must be non-NULL and 16-byte aligned";
  if (grad_ld < c.P || grad_ld % 4 != 0) return "grad_ld must be >= P and a multiple of 4";
  if (accumulate != 0 && accumulate != 1) return "accumulate must be 0 or 1";
  return "";
}

std::string check_workspace(const void* p, size_t have, size_t need) {
  if (need == 0) return "";
  if (!p || reinterpret_cast<uintptr_t>(p) % 256 != 0) return "workspace must be non-NULL and 256-byte aligned";
  if (have < need) return format("workspace of %zu bytes, %zu needed", have, need);
  return "";
}

#define CHECK(c, call)                                                  \
  do {                                                                  \
    const std::string e_ = (call);                                      \
    if (!e_.empty()) return fail((c), GASLOC_EINVAL, e_);               \
  } while (0)

LiveRows live_rows(const gasloc_ctx& c) {
  LiveRows w{c.buf.x, c.buf.y, c.buf.ld, 0};
  for (int i = 0; i < c.n; ++i)
    if (c.stepped[static_cast<size_t>(i)]) w.stepped |= 1ull << i;
  return w;
}

Spans row_spans(int n, const int64_t* row_ptr) {
  Spans s{};
  for (int i = 0; i <= n; ++i) s.begin[i] = static_cast<int32_t>(row_ptr[i]);
  return s;
}

// Consecutive items of `per` rows each, none of them over two workers.
Spans item_spans(int n, const int64_t* row_ptr, int64_t per) {
  Spans s{};
  for (int i = 0; i < n; ++i)
    s.begin[i + 1] = s.begin[i] + static_cast<int32_t>((row_ptr[i + 1] - row_ptr[i] + per - 1) / per);
  return s;
}

bool whole_vectors(int64_t cols, int32_t dtype) { return cols % (dtype == GASLOC_BF16 ? 8 : 4) == 0; }

// Rows of `cols` elements that begin on 16-byte boundaries and are whole 16-byte vectors.
bool vector_rows(const void* p, int64_t ld, int64_t cols, int32_t dtype) {
  return aligned16(p) && whole_vectors(ld, dtype) && whole_vectors(cols, dtype);
}

// The same for a weight at column `begin` of the parameters and of the gradients.
bool vector_columns(const gasloc_ctx& c, int64_t begin) {
  return begin * static_cast<int64_t>(param_bytes(c.hp.param_dtype)) % 16 == 0;
}

size_t round256(size_t bytes) { return (bytes + 255) / 256 * 256; }

// ---------------------------------------------------------------------------
// embedding
// ---------------------------------------------------------------------------

// Sorted entries per workgroup of the sums: a power of two from 8 to 32, with which the rows make at least about two
// workgroups per CU (256 of them) while there are enough.
int64_t sum_chunk(int64_t rows) {
  int64_t chunk = 32;
  while (chunk > 8 && rows / chunk < 512) chunk /= 2;
  return chunk;
}

struct EmbeddingSpace {
  size_t keys[2], pos[2], partial, bytes;
};

EmbeddingSpace embedding_space(int n, int32_t width, const int64_t* row_ptr) {
  const size_t rows = static_cast<size_t>(row_ptr[n]);
  int64_t longest = 0;
  for (int i = 0; i < n; ++i) longest = std::max(longest, row_ptr[i + 1] - row_ptr[i]);
  const Spans chunks = item_spans(n, row_ptr, sum_chunk(row_ptr[n]));
  EmbeddingSpace s{};
  size_t at = 0;
  const auto take = [&](size_t bytes) {
    const size_t here = at;
    at += round256(bytes);
    return here;
  };
  const bool merges = longest > gasloc::kSortTile;
  for (int k = 0; k < 2; ++k) {
    s.keys[k] = k == 0 || merges ? take(4 * rows) : s.keys[0];
    s.pos[k] = k == 0 || merges ? take(4 * rows) : s.pos[0];
  }
  s.partial = take(sizeof(float) * 2 * static_cast<size_t>(chunks.begin[n]) * static_cast<size_t>(width));
  s.bytes = at;
  return s;
}

std::string check_table(const gasloc_ctx& c, int64_t begin, int32_t vocab, int32_t width, float scale) {
  if (vocab < 1 || vocab > (1 << 24)) return "vocab must be in [1, 2^24]";
  if (width < 1) return "width must be >= 1";
  if (!std::isfinite(scale)) return "scale must be finite";
  return check_columns(c, "table", begin, static_cast<int64_t>(vocab) * width);
}

// ---------------------------------------------------------------------------
// layer norm
// ---------------------------------------------------------------------------

std::string check_norm(const gasloc_ctx& c, int64_t gain, int64_t bias, int32_t width) {
  if (width < 1 || width > gasloc::kMaxNormWidth) return "width must be in [1, 16384]";
  std::string e = check_columns(c, "gain", gain, width);
  if (e.empty() && bias >= 0) e = check_columns(c, "bias", bias, width);
  if (e.empty() && bias >= 0 && std::llabs(gain - bias) < width) e = "gain and bias overlap";
  return e;
}

// Rows per workgroup: enough that about `target` workgroups share the rows, a
// multiple of the rows that its waves take at a time.
int64_t norm_tile_rows(int64_t rows, int waves, int64_t target) {
  const int64_t at_once = waves == 1 ? 4 : 1;
  const int64_t per = (rows + target - 1) / target;
  return std::min<int64_t>(1024, std::max<int64_t>(1, (per + at_once - 1) / at_once) * at_once);
}

// Forward: 4 rows per wave of a workgroup keep the weights' reads small beside the rows.
int64_t forward_tile_rows(const gasloc_ctx& c, int64_t rows, int waves) {
  return std::min<int64_t>(16, norm_tile_rows(rows, waves, 4 * c.cus));
}

// Backward: about four workgroups per CU, each of which leaves two rows of partial sums.
int64_t backward_tile_rows(const gasloc_ctx& c, int64_t rows, int waves) {
  return norm_tile_rows(rows, waves, 4 * c.cus);
}

// ---------------------------------------------------------------------------
// linear
// ---------------------------------------------------------------------------

constexpr int32_t kMaxFeatures = 1 << 20;

std::string check_weight(const gasloc_ctx& c, int64_t weight, int32_t out_features, int32_t in_features) {
  if (out_features < 1 || out_features > kMaxFeatures || in_features < 1 || in_features > kMaxFeatures)
    return "features must be in [1, 2^20]";
  return check_columns(c, "weight", weight, static_cast<int64_t>(out_features) * in_features);
}

// Workgroups of every worker's product with tiles of `tile` outputs, in one part each.
// The weight's gradient begins with the workers that have the most rows, whose tiles take longest.
// False if there are too many for one launch.
bool linear_tiles(int n, const int64_t* row_ptr, gasloc::LinearPass pass, int tile, gasloc::LinearArgs* a) {
  const auto cut = [tile](int64_t v) { return (v + tile - 1) / tile; };
  for (int i = 0; i < n; ++i) a->order[i] = static_cast<uint8_t>(i);
  if (pass == gasloc::kLinearWeight)
    std::stable_sort(a->order, a->order + n, [&](int i, int j) {
      return row_ptr[i + 1] - row_ptr[i] > row_ptr[j + 1] - row_ptr[j];
    });
  a->chunk = 0;
  int64_t at = 0;
  for (int i = 0; i < n; ++i) {
    const int64_t rows = row_ptr[i + 1] - row_ptr[i];
    at += pass == gasloc::kLinearWeight    ? cut(a->out_features) * cut(a->in_features)
          : pass == gasloc::kLinearForward ? cut(rows) * cut(a->out_features)
                                           : cut(rows) * cut(a->in_features);
    if (at > kMaxGroups) return false;
    a->tiles.begin[i + 1] = static_cast<int32_t>(at);
    a->parts.begin[i + 1] = i + 1;
  }
  return true;
}

// The length of a worker's sums.
int64_t depth_of(const gasloc::LinearArgs& a, const int64_t* row_ptr, gasloc::LinearPass pass, int worker) {
  return pass == gasloc::kLinearForward ? a.in_features
         : pass == gasloc::kLinearInput ? a.out_features
                                        : row_ptr[worker + 1] - row_ptr[worker];
}

// All outputs of the product.
int64_t outputs_of(int n, const gasloc::LinearArgs& a, const int64_t* row_ptr, gasloc::LinearPass pass) {
  return pass == gasloc::kLinearWeight ? static_cast<int64_t>(n) * a.out_features * a.in_features
                                       : row_ptr[n] * (pass == gasloc::kLinearForward ? a.out_features : a.in_features);
}

// Whether a product in bf16 takes less time in `large` tiles of 256 than in `small` ones of 128.  The first fill a CU
// each, of the second two go on a CU: a round of large tiles takes 1.65 times as long as one of pairs of small ones,
// which takes 1/0.65 times as long as one of single ones.  Asked below two rounds of large tiles, which are taken from
// there on (they read half as much).  1024 -> 1024, n = 8, large /
// small tiles: 2048 rows each (256 / 1024 tiles) 34 / 41 us, 1024 rows (128 / 512) 29 / 23.
bool large_tiles(const gasloc_ctx& c, int64_t large, int64_t small) {
  const int64_t rounds = (large + c.cus - 1) / c.cus, per_cu = (small + c.cus - 1) / c.cus;
  return 33 * rounds <= 20 * (per_cu / 2) + 13 * (per_cu % 2);
}

// Cuts a product that tiles of 256 do not suit into tiles of 128 outputs, or of 64 where those would be too few for
// the CUs (fewer than one per CU, or two in F32, whose matrix instructions take longer) and none would have many steps
// to do (20 per CU in BF16, 128 in F32): such products wait for their loads, not for the matrix cores.  Others keep the
// tiles of 128, which read half as much for an output.  Tiles of 128 / of 64, bf16: n = 4, 256 rows each, 512 -> 512
// 7.9 / 5.4 us; n = 16, 512 rows, 512 -> 512 9.2 / 11.7; the weight's gradient of n = 4, 4096 rows, 512 -> 512 25 / 29;
// fp32: n = 4, 256 rows, 512 -> 512 35 / 13.  Returns the side, 0 if the product is too large.
int cut_linear(const gasloc_ctx& c, const int64_t* row_ptr, gasloc::LinearPass pass, int32_t dtype,
               gasloc::LinearArgs* a) {
  if (!linear_tiles(c.n, row_ptr, pass, 128, a)) return 0;
  const bool f32 = dtype == GASLOC_F32;
  const int64_t full = static_cast<int64_t>(c.cus) * (128 * 128);  // outputs of one tile per CU
  const int64_t products = row_ptr[c.n] * a->in_features;          // times out_features
  if (outputs_of(c.n, *a, row_ptr, pass) >= (f32 ? 2 : 1) * full ||
      products >= (f32 ? 128 * 16 : 20 * 32) * full / a->out_features)
    return 128;
  linear_tiles(c.n, row_ptr, pass, 64, a);
  return 64;
}

// Splits the sums of a product whose tiles are fewer than two per CU, so that about two workgroups per CU share the
// steps of k, if that saves more steps than the parts cost: the join's launch takes about as long as 16 steps (4 us),
// and writing and adding a megabyte of parts as 2.  bf16, whole / split: n = 2, 64 rows each, 8192 -> 512 40 / 14 us;
// n = 16, 64 rows, 1024 -> 1024 9.4 / 14.  Tiles are counted whatever they cost: a weight's gradient with most rows in
// one worker is not split, and few CUs have its work (n = 8, 2048 -> 2048, 30011 rows, 95% of them in one worker: 622
// us, spread evenly 245).  Returns the bytes of the parts.
size_t split_linear(const gasloc_ctx& c, const int64_t* row_ptr, gasloc::LinearPass pass, int32_t dtype,
                    gasloc::LinearArgs* a) {
  const int n = c.n;
  const int64_t total = a->tiles.begin[n], want = 2 * static_cast<int64_t>(c.cus);
  if (total == 0 || total >= want) return 0;
  const int64_t per_step = gasloc::kLinearStep / static_cast<int64_t>(param_bytes(dtype));
  int64_t tiles[gasloc::kMaxReplicas], steps[gasloc::kMaxReplicas], work = 0, longest = 0;
  for (int i = 0; i < n; ++i) {
    tiles[i] = a->tiles.begin[i + 1] - a->tiles.begin[i];
    steps[i] = (depth_of(*a, row_ptr, pass, a->order[i]) + per_step - 1) / per_step;
    work += tiles[i] * steps[i];
    if (tiles[i] > 0) longest = std::max(longest, steps[i]);
  }
  const int64_t part = std::max<int64_t>(4, ((work + want - 1) / want + 3) / 4 * 4);
  const auto parts_of = [&](int i) { return std::max<int64_t>(1, (steps[i] + part - 1) / part); };
  int64_t all_parts = 0;
  for (int i = 0; i < n; ++i) all_parts += parts_of(i);
  const int64_t outputs = outputs_of(n, *a, row_ptr, pass);
  const size_t bytes = sizeof(float) * static_cast<size_t>(pass == gasloc::kLinearWeight ? outputs / n * all_parts
                                                                                          : outputs * parts_of(0));
  if (longest - part < 16 + 2 * static_cast<int64_t>(bytes >> 20)) return 0;
  a->chunk = static_cast<int32_t>(part * per_step);
  for (int i = 0; i < n; ++i) {
    a->tiles.begin[i + 1] = static_cast<int32_t>(a->tiles.begin[i] + tiles[i] * parts_of(i));
    a->parts.begin[i + 1] = static_cast<int32_t>(a->parts.begin[i] + parts_of(i));
  }
  return bytes;
}

gasloc_status run_linear(gasloc_ctx* c, gasloc::LinearArgs* a, gasloc::LinearPass pass, const int64_t* row_ptr,
                         int32_t dtype, void* workspace, size_t workspace_bytes) {
  a->w = live_rows(*c);
  a->n = c->n;
  a->rows = row_spans(c->n, row_ptr);
  const bool vec = vector_columns(*c, a->weight) && (!a->x || vector_rows(a->x, a->x_ld, a->in_features, dtype)) &&
                   (!a->dout || vector_rows(a->dout, a->dout_ld, a->out_features, dtype)) &&
                   (!a->out || vector_rows(a->out, a->out_ld, 0, dtype)) && a->in_features % 8 == 0 &&
                   a->out_features % 8 == 0;
  int64_t most = 0;
  for (int i = 0; i < c->n; ++i) most = std::max(most, row_ptr[i + 1] - row_ptr[i]);
  int tile = vec && dtype == GASLOC_BF16 ? 256 : 128;
  // Few rows: the weights' way through LDS in tiles of 128 outputs leaves too few loads in flight (n = 16, one row
  // each, 2048 -> 2048, bf16 rows, fp32 weights: 61 us against 48).  One worker with more rows than the others sends
  // all of them to the tiles, which costs nothing there: 15 of one row and one of 16 take 43 us, one of 17 40.
  if (pass == gasloc::kLinearForward && most <= gasloc::kFewRows) tile = gasloc::kFewRows;
  bool fits = linear_tiles(c->n, row_ptr, pass, tile, a);
  const int64_t large = a->tiles.begin[c->n];
  if (tile == 256 && fits && large < 2 * c->cus) {
    linear_tiles(c->n, row_ptr, pass, 128, a);
    if (large_tiles(*c, large, a->tiles.begin[c->n]))
      linear_tiles(c->n, row_ptr, pass, 256, a);
    else
      tile = 128;
  }
  if (tile == 128) {
    tile = cut_linear(*c, row_ptr, pass, dtype, a);
    fits = tile != 0;
  }
  if (!fits) return fail(c, GASLOC_EINVAL, "product too large for one launch");
  if (a->tiles.begin[c->n] == 0) return GASLOC_OK;
  if (tile == 128 || tile == 64) {
    CHECK(c, check_workspace(workspace, workspace_bytes, split_linear(*c, row_ptr, pass, dtype, a)));
    a->partial = static_cast<float*>(workspace);
  }
  DeviceGuard guard(c->device);
  HIP_TRY(c, gasloc::launch_linear(*a, pass, c->hp.param_dtype, dtype, tile, vec, c->stream));
  return GASLOC_OK;
}

}  // namespace

extern "C" {

gasloc_status gasloc_embedding(gasloc_ctx* c, int64_t begin, int32_t vocab, int32_t width, float scale,
                               const int64_t* row_ptr, const int32_t* tokens, int32_t dtype, void* out,
                               int64_t out_ld) {
  return guarded([&] {
    const gasloc_status st = check_context(c);
    if (st != GASLOC_OK) return st;
    CHECK(c, check_table(*c, begin, vocab, width, scale));
    CHECK(c, check_rows(c->n, row_ptr));
    CHECK(c, check_types(*c, dtype));
    const int64_t rows = row_ptr[c->n];
    CHECK(c, check_act("out", out, out_ld, width, rows, dtype));
    if (rows > 0 && (!tokens || reinterpret_cast<uintptr_t>(tokens) % 4 != 0))
      return fail(c, GASLOC_EINVAL, "tokens must be non-NULL and 4-byte aligned");
    if (rows == 0) return GASLOC_OK;
    gasloc::EmbeddingArgs a{};
    a.w = live_rows(*c);
    a.begin = begin;
    a.vocab = vocab;
    a.width = width;
    a.scale = scale;
    a.n = c->n;
    a.tokens = tokens;
    a.out = out;
    a.out_ld = out_ld;
    a.rows = row_spans(c->n, row_ptr);
    DeviceGuard guard(c->device);
    HIP_TRY(c, gasloc::launch_embedding(a, c->hp.param_dtype, dtype, c->stream));
    return GASLOC_OK;
  });
}

gasloc_status gasloc_embedding_grad_workspace(const gasloc_ctx* c, int32_t width, const int64_t* row_ptr,
                                              size_t* bytes) {
  return guarded([&] {
    if (!c || !bytes) return fail(nullptr, GASLOC_EINVAL, "NULL argument");
    if (width < 1) return fail(nullptr, GASLOC_EINVAL, "width must be >= 1");
    CHECK(nullptr, check_rows(c->n, row_ptr));
    *bytes = embedding_space(c->n, width, row_ptr).bytes;
    return GASLOC_OK;
  });
}

gasloc_status gasloc_embedding_grad(gasloc_ctx* c, int64_t begin, int32_t vocab, int32_t width, float scale,
                                    const int64_t* row_ptr, const int32_t* tokens, int32_t dtype, const void* dout,
                                    int64_t dout_ld, float* grads, int64_t grad_ld, int32_t accumulate,
                                    void* workspace, size_t workspace_bytes) {
  return guarded([&] {
    const gasloc_status st = check_context(c);
    if (st != GASLOC_OK) return st;
    const int n = c->n;
    CHECK(c, check_table(*c, begin, vocab, width, scale));
    CHECK(c, check_rows(n, row_ptr));
    CHECK(c, check_types(*c, dtype));
    const int64_t rows = row_ptr[n];
    CHECK(c, check_act("dout", dout, dout_ld, width, rows, dtype));
    CHECK(c, check_grads(*c, grads, grad_ld, accumulate));
    if (rows > 0 && (!tokens || reinterpret_cast<uintptr_t>(tokens) % 4 != 0))
      return fail(c, GASLOC_EINVAL, "tokens must be non-NULL and 4-byte aligned");
    const EmbeddingSpace space = embedding_space(n, width, row_ptr);
    CHECK(c, check_workspace(workspace, workspace_bytes, space.bytes));
    if (rows == 0 && accumulate) return GASLOC_OK;
    // Rows without tokens are zeroed about 16 KB to a workgroup (or four rows), in the order of the rows: what is
    // written at any time is one stretch of memory (n = 16 tables of 32000 x 1024, 1 MB each: 454 us; 256 KB: 436;
    // 16 KB: 358).
    const int64_t fill_rows = std::min<int64_t>(gasloc::kMaxChunk, std::max<int64_t>(4, 4096 / width));
    const int64_t chunk = sum_chunk(rows);
    const Spans chunks = item_spans(n, row_ptr, chunk);
    CHECK(c, check_launch("table", chunks.begin[n] + (accumulate ? 0 : n * ((vocab + fill_rows - 1) / fill_rows)), 256));
    char* ws = static_cast<char*>(workspace);
    const auto keys = [&](int k) { return reinterpret_cast<uint32_t*>(ws + space.keys[k]); };
    const auto pos = [&](int k) { return reinterpret_cast<int32_t*>(ws + space.pos[k]); };
    DeviceGuard guard(c->device);
    int cur = 0;
    if (rows > 0) {
      gasloc::SortArgs s{};
      s.tokens = tokens;
      s.vocab = vocab;
      s.n = n;
      while (s.key_bits < 32 && (static_cast<uint32_t>(vocab) >> s.key_bits) != 0) ++s.key_bits;
      s.keys = keys(0);
      s.pos = pos(0);
      s.rows = row_spans(n, row_ptr);
      s.tiles = item_spans(n, row_ptr, gasloc::kSortTile);
      HIP_TRY(c, gasloc::launch_token_sort(s, c->stream));
      int64_t longest = 0;
      for (int i = 0; i < n; ++i) longest = std::max(longest, row_ptr[i + 1] - row_ptr[i]);
      for (int64_t run = gasloc::kSortTile; run < longest; run *= gasloc::kMergeWays, cur ^= 1) {
        gasloc::MergeArgs m{};
        m.keys = keys(cur);
        m.pos = pos(cur);
        m.keys_out = keys(cur ^ 1);
        m.pos_out = pos(cur ^ 1);
        m.run = run;
        m.n = n;
        m.rows = s.rows;
        m.blocks = item_spans(n, row_ptr, 256);
        HIP_TRY(c, gasloc::launch_token_merge(m, c->stream));
      }
    }
    gasloc::EmbeddingGradArgs a{};
    a.keys = keys(cur);
    a.pos = pos(cur);
    a.dout = dout;
    a.dout_ld = dout_ld;
    a.grads = grads;
    a.grad_ld = grad_ld;
    a.begin = begin;
    a.partial = reinterpret_cast<float*>(ws + space.partial);
    a.scale = scale;
    a.vocab = vocab;
    a.width = width;
    a.n = n;
    a.chunk = static_cast<int32_t>(chunk);
    a.accumulate = accumulate;
    a.rows = row_spans(n, row_ptr);
    a.chunks = chunks;
    a.fill_rows = static_cast<int32_t>(fill_rows);
    HIP_TRY(c, gasloc::launch_embedding_sums(a, dtype, c->stream));
    if (rows > a.chunk) HIP_TRY(c, gasloc::launch_embedding_join(a, c->stream));
    return GASLOC_OK;
  });
}

gasloc_status gasloc_layer_norm(gasloc_ctx* c, int64_t gain, int64_t bias, int32_t width, float eps,
                                const int64_t* row_ptr, const void* x, int64_t x_ld, int32_t dtype, void* out,
                                int64_t out_ld, float* stats) {
  return guarded([&] {
    const gasloc_status st = check_context(c);
    if (st != GASLOC_OK) return st;
    CHECK(c, check_norm(*c, gain, bias, width));
    if (!(std::isfinite(eps) && eps > 0.0f)) return fail(c, GASLOC_EINVAL, "eps must be finite and > 0");
    CHECK(c, check_rows(c->n, row_ptr));
    CHECK(c, check_types(*c, dtype));
    const int64_t rows = row_ptr[c->n];
    CHECK(c, check_act("x", x, x_ld, width, rows, dtype));
    CHECK(c, check_act("out", out, out_ld, width, rows, dtype));
    CHECK(c, check_in_place("out", out, out_ld, x, x_ld));
    if (reinterpret_cast<uintptr_t>(stats) % 8 != 0) return fail(c, GASLOC_EINVAL, "stats must be 8-byte aligned");
    if (rows == 0) return GASLOC_OK;
    gasloc::NormArgs a{};
    a.w = live_rows(*c);
    a.gain = gain;
    a.bias = bias < 0 ? -1 : bias;
    a.width = width;
    a.n = c->n;
    a.eps = eps;
    a.x = x;
    a.x_ld = x_ld;
    a.out = out;
    a.out_ld = out_ld;
    a.stats = stats;
    a.tile_rows = static_cast<int32_t>(forward_tile_rows(*c, rows, gasloc::norm_waves(width)));
    a.rows = row_spans(c->n, row_ptr);
    a.tiles = item_spans(c->n, row_ptr, a.tile_rows);
    CHECK(c, check_launch("rows", a.tiles.begin[c->n], std::max(4, gasloc::norm_waves(width)) * 64));
    DeviceGuard guard(c->device);
    HIP_TRY(c, gasloc::launch_layer_norm(a, c->hp.param_dtype, dtype, whole_vectors(width, dtype), c->stream));
    return GASLOC_OK;
  });
}

gasloc_status gasloc_layer_norm_grad_workspace(const gasloc_ctx* c, int32_t width, const int64_t* row_ptr,
                                               size_t* bytes) {
  return guarded([&] {
    if (!c || !bytes) return fail(nullptr, GASLOC_EINVAL, "NULL argument");
    if (width < 1 || width > gasloc::kMaxNormWidth) return fail(nullptr, GASLOC_EINVAL, "width must be in [1, 16384]");
    CHECK(nullptr, check_rows(c->n, row_ptr));
    const int64_t per = backward_tile_rows(*c, row_ptr[c->n], gasloc::norm_waves(width));
    const Spans tiles = item_spans(c->n, row_ptr, per);
    *bytes = round256(sizeof(float) * 2 * static_cast<size_t>(tiles.begin[c->n]) * static_cast<size_t>(width));
    return GASLOC_OK;
  });
}

gasloc_status gasloc_layer_norm_grad(gasloc_ctx* c, int64_t gain, int64_t bias, int32_t width,
                                     const int64_t* row_ptr, const void* x, int64_t x_ld, const float* stats,
                                     const void* dout, int64_t dout_ld, int32_t dtype, void* dx, int64_t dx_ld,
                                     float* grads, int64_t grad_ld, int32_t accumulate, void* workspace,
                                     size_t workspace_bytes) {
  return guarded([&] {
    const gasloc_status st = check_context(c);
    if (st != GASLOC_OK) return st;
    CHECK(c, check_norm(*c, gain, bias, width));
    CHECK(c, check_rows(c->n, row_ptr));
    CHECK(c, check_types(*c, dtype));
    const int64_t rows = row_ptr[c->n];
    CHECK(c, check_act("x", x, x_ld, width, rows, dtype));
    CHECK(c, check_act("dout", dout, dout_ld, width, rows, dtype));
    CHECK(c, check_act("dx", dx, dx_ld, width, rows, dtype));
    CHECK(c, check_in_place("dx", dx, dx_ld, dout, dout_ld));
    CHECK(c, check_in_place("dx", dx, dx_ld, x, x_ld));
    if ((rows > 0 && !stats) || reinterpret_cast<uintptr_t>(stats) % 8 != 0)
      return fail(c, GASLOC_EINVAL, "stats must be non-NULL and 8-byte aligned");
    CHECK(c, check_grads(*c, grads, grad_ld, accumulate));
    size_t need = 0;
    const gasloc_status sized = gasloc_layer_norm_grad_workspace(c, width, row_ptr, &need);
    if (sized != GASLOC_OK) return sized;
    CHECK(c, check_workspace(workspace, workspace_bytes, need));
    if (rows == 0 && accumulate) return GASLOC_OK;
    gasloc::NormGradArgs a{};
    a.w = live_rows(*c);
    a.gain = gain;
    a.bias = bias < 0 ? -1 : bias;
    a.width = width;
    a.n = c->n;
    a.accumulate = accumulate;
    a.x = x;
    a.x_ld = x_ld;
    a.stats = stats;
    a.dout = dout;
    a.dout_ld = dout_ld;
    a.dx = dx;
    a.dx_ld = dx_ld;
    a.partial = static_cast<float*>(workspace);
    a.grads = grads;
    a.grad_ld = grad_ld;
    a.tile_rows = static_cast<int32_t>(backward_tile_rows(*c, rows, gasloc::norm_waves(width)));
    a.rows = row_spans(c->n, row_ptr);
    a.tiles = item_spans(c->n, row_ptr, a.tile_rows);
    DeviceGuard guard(c->device);
    if (rows > 0)
      HIP_TRY(c, gasloc::launch_layer_norm_grad(a, c->hp.param_dtype, dtype, whole_vectors(width, dtype), c->stream));
    HIP_TRY(c, gasloc::launch_layer_norm_join(a, c->stream));
    return GASLOC_OK;
  });
}

gasloc_status gasloc_linear(gasloc_ctx* c, int64_t weight, int32_t out_features, int32_t in_features,
                            const int64_t* row_ptr, const void* x, int64_t x_ld, int32_t dtype, void* out,
                            int64_t out_ld, void* workspace, size_t workspace_bytes) {
  return guarded([&] {
    const gasloc_status st = check_context(c);
    if (st != GASLOC_OK) return st;
    CHECK(c, check_weight(*c, weight, out_features, in_features));
    CHECK(c, check_rows(c->n, row_ptr));
    CHECK(c, check_types(*c, dtype));
    CHECK(c, check_act("x", x, x_ld, in_features, row_ptr[c->n], dtype));
    CHECK(c, check_act("out", out, out_ld, out_features, row_ptr[c->n], dtype));
    gasloc::LinearArgs a{};
    a.weight = weight;
    a.out_features = out_features;
    a.in_features = in_features;
    a.x = x;
    a.x_ld = x_ld;
    a.out = out;
    a.out_ld = out_ld;
    return run_linear(c, &a, gasloc::kLinearForward, row_ptr, dtype, workspace, workspace_bytes);
  });
}

gasloc_status gasloc_linear_grad_input(gasloc_ctx* c, int64_t weight, int32_t out_features, int32_t in_features,
                                       const int64_t* row_ptr, const void* dout, int64_t dout_ld, int32_t dtype,
                                       void* dx, int64_t dx_ld, void* workspace, size_t workspace_bytes) {
  return guarded([&] {
    const gasloc_status st = check_context(c);
    if (st != GASLOC_OK) return st;
    CHECK(c, check_weight(*c, weight, out_features, in_features));
    CHECK(c, check_rows(c->n, row_ptr));
    CHECK(c, check_types(*c, dtype));
    CHECK(c, check_act("dout", dout, dout_ld, out_features, row_ptr[c->n], dtype));
    CHECK(c, check_act("dx", dx, dx_ld, in_features, row_ptr[c->n], dtype));
    gasloc::LinearArgs a{};
    a.weight = weight;
    a.out_features = out_features;
    a.in_features = in_features;
    a.dout = dout;
    a.dout_ld = dout_ld;
    a.out = dx;
    a.out_ld = dx_ld;
    return run_linear(c, &a, gasloc::kLinearInput, row_ptr, dtype, workspace, workspace_bytes);
  });
}

gasloc_status gasloc_linear_workspace(const gasloc_ctx* c, int32_t out_features, int32_t in_features,
                                      const int64_t* row_ptr, int32_t dtype, size_t* bytes) {
  return guarded([&] {
    if (!c || !bytes) return fail(nullptr, GASLOC_EINVAL, "NULL argument");
    if (out_features < 1 || out_features > kMaxFeatures || in_features < 1 || in_features > kMaxFeatures)
      return fail(nullptr, GASLOC_EINVAL, "features must be in [1, 2^20]");
    CHECK(nullptr, check_rows(c->n, row_ptr));
    CHECK(nullptr, check_types(*c, dtype));
    *bytes = 0;
    for (gasloc::LinearPass pass : {gasloc::kLinearForward, gasloc::kLinearInput, gasloc::kLinearWeight}) {
      gasloc::LinearArgs a{};
      a.out_features = out_features;
      a.in_features = in_features;
      if (cut_linear(*c, row_ptr, pass, dtype, &a) != 0)
        *bytes = std::max(*bytes, split_linear(*c, row_ptr, pass, dtype, &a));
    }
    *bytes = round256(*bytes);
    return GASLOC_OK;
  });
}

gasloc_status gasloc_linear_grad_weight(gasloc_ctx* c, int64_t weight, int32_t out_features, int32_t in_features,
                                        const int64_t* row_ptr, const void* x, int64_t x_ld, const void* dout,
                                        int64_t dout_ld, int32_t dtype, float* grads, int64_t grad_ld,
                                        int32_t accumulate, void* workspace, size_t workspace_bytes) {
  return guarded([&] {
    const gasloc_status st = check_context(c);
    if (st != GASLOC_OK) return st;
    CHECK(c, check_weight(*c, weight, out_features, in_features));
    CHECK(c, check_rows(c->n, row_ptr));
    CHECK(c, check_types(*c, dtype));
    CHECK(c, check_act("x", x, x_ld, in_features, row_ptr[c->n], dtype));
    CHECK(c, check_act("dout", dout, dout_ld, out_features, row_ptr[c->n], dtype));
    CHECK(c, check_grads(*c, grads, grad_ld, accumulate));
    if (row_ptr[c->n] == 0 && accumulate) return GASLOC_OK;
    gasloc::LinearArgs a{};
    a.weight = weight;
    a.out_features = out_features;
    a.in_features = in_features;
    a.x = x;
    a.x_ld = x_ld;
    a.dout = dout;
    a.dout_ld = dout_ld;
    a.grads = grads;
    a.grad_ld = grad_ld;
    a.accumulate = accumulate;
    return run_linear(c, &a, gasloc::kLinearWeight, row_ptr, dtype, workspace, workspace_bytes);
  });
}

}  // extern "C"
