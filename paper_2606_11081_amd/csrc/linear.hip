// Linear layers of every worker on the matrix cores: for each worker
//   forward  out = x W^T,  input  dx = dout W,  weight  dW = dout^T x,
// all of the form C[m][n] = sum_k A(m, k) B(n, k).
//
// A workgroup makes one tile of C: 256 x 256 outputs by eight waves (bf16), or
// 128 x 128 or 64 x 64 by four; 64 bytes of k of both operands at a time (a step) pass
// through four buffers in LDS, with the loads of what follows in flight in
// registers (fp32 weights that meet bf16 activations are rounded on the way).
// An operand whose rows run along k lies in LDS as [row][k] and is read in
// 16-byte fragments; one whose rows run across k lies as [k][row] and is
// transposed by the LDS read itself (bf16) or read by words (fp32).
//
// Measured on several cards, bf16 rows: n = 16, 32768 rows, 1024 -> 4096, bf16
// weights 270 to 278 us (990 to 1020 TFLOP/s); input gradient of 2048 -> 2048 under
// fp32 weights 264 to 280 us (980 to 1040); weight gradient of n = 8, 30011 ragged
// rows 227 to 240 us (1050 to 1110).  fp32, n = 4, 1024 rows each, 2048 -> 2048: 257
// to 261 us in each direction (132 to 134 TFLOP/s).  Small products wait
// for their first loads and the launches: n = 8, 256 rows each, 1024 -> 1024 in bf16
// 11 us; weight gradient of n = 3, 1111 rows, 513 x 257 in fp32 15 us, in two launches.  A 2048-deep loop
// alone runs at 1100 to 1200.  The loads bound it: without those of the loop it
// ran at 1340 to 1510, with all of them hitting L2 at 1230 to 1330, while the
// place of stores, loads and waits among the products changes less than 2%.  A
// tile's first loads and its stores, 6 us of a 1024-deep tile's 34, overlap
// nothing, since one workgroup fills a CU; loading the next tile's beginning
// before storing needs more registers than there are.
#pragma clang fp contract(off)

#include <type_traits>

#include "layers_device.h"

namespace gasloc {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kBuffers = 4;
constexpr uint32_t kNowhere = 0x80000000u;  // no window holds this offset or one behind it: the load gives zeros

// A range of memory of at most 2^31 bytes that loads are checked against; what lies outside reads as zero.
// (Both are the same in every lane; left to find that out, the compiler loops over the lanes' values.)
__device__ __forceinline__ __amdgpu_buffer_rsrc_t window(const void* p, uint32_t bytes) {
  const uint64_t at = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(at));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(at >> 32));
  p = reinterpret_cast<const void*>(static_cast<uint64_t>(hi) << 32 | lo);
  bytes = __builtin_amdgcn_readfirstlane(bytes);
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, static_cast<int>(bytes), 0x00027000);
}

template <typename T>
__device__ __forceinline__ __attribute__((address_space(3))) T* lds_pointer(uint32_t at) {
  return (__attribute__((address_space(3))) T*)static_cast<uintptr_t>(at);
}

// One operand of a workgroup's tile: ROWS rows (of m or n), KT of k per step.
// KC: rows run along k in memory.  ST: type in memory, CT: type of the product.
// VEC: 16-byte chunks lie on 16-byte boundaries and are inside or outside as a whole.
//
// Rows are loaded by whole 128-byte lines, which along k may be two steps at
// once (64 bytes at a time take twice the requests to L2, which were what
// bounded the loop).
//
// In LDS a KC step is [row][64 bytes], its four blocks of 16 permuted by the
// row's place among sixteen; other bf16 steps are [k][row], blocks of 32 bytes
// permuted by k; fp32 ones have their lines 16 bytes apart.  So the lanes that a
// fragment read serves at a time do not meet in a bank (plain padding of 16 bytes
// per KC row cost as many cycles in conflicts again).  Conflicts remain: 31% of the
// LDS cycles of a forward pass, 18% of an input gradient's, 1% of a weight gradient's,
// so most of them come with the writes of KC operands.
template <int ROWS, int THREADS, bool KC, int ST, int CT, bool VEC>
struct Operand {
  static constexpr int kSize = CT == GASLOC_BF16 ? 2 : 4;  // bytes of an element in LDS
  static constexpr int kSrc = ST == GASLOC_BF16 ? 2 : 4;   // and in memory
  static constexpr int KT = 64 / kSize;                    // k per step
  static constexpr int kSpan = KC && ST == CT ? 2 : 1;     // steps per load
  static constexpr int E = 16 / kSrc;                      // elements of a chunk: 16 bytes in memory
  static constexpr int kAcross = KC ? 8 : ROWS / E;        // chunks of a line in memory
  static constexpr int kLines = THREADS / kAcross;         // lines between a thread's chunks
  static constexpr int kChunks = (KC ? ROWS : KT) / kLines;
  static constexpr int kStride = KC ? 64 : ROWS * kSize + (CT == GASLOC_BF16 ? 0 : 16);
  static constexpr int kLds = KC ? ROWS * kStride : KT * kStride;

  const char* at;  // row 0 of the load to come
  int left;        // k from there on
  int64_t ahead;   // bytes to the load after it
  uint32_t line;   // bytes between lines in memory
  int rows;        // rows inside (of ROWS)
  uint32_t full;   // bytes of a whole load (not KC) or of the rows from `at` on (KC)
  uint32_t off;    // of chunk 0 of this thread
  typedef uint32_t Words[kChunks][4];  // a load on its way to LDS

  // p: element (first, 0) of the operand; `rows_left` rows from there on exist
  __device__ __forceinline__ void start(const void* p, int64_t ld, int rows_left, int k) {
    at = static_cast<const char*>(p);
    line = static_cast<uint32_t>(ld * kSrc);
    rows = rows_left < ROWS ? rows_left : ROWS;
    left = k;
    ahead = KC ? kSpan * KT * kSrc : KT * static_cast<int64_t>(line);
    full = KC ? static_cast<uint32_t>(rows - 1) * line + static_cast<uint32_t>(k) * kSrc
              : static_cast<uint32_t>(KT - 1) * line + static_cast<uint32_t>(rows) * kSrc;
    off = static_cast<uint32_t>(line_of(0)) * line + static_cast<uint32_t>(col_of() * kSrc);
    if (!KC && VEC && col_of() >= rows) off = kNowhere;
  }
  // The chunk j of this thread: its line in memory (a row of m or n, or of k) and its first column.
  __device__ __forceinline__ int line_of(int j) const { return static_cast<int>(threadIdx.x) / kAcross + kLines * j; }
  __device__ __forceinline__ int col_of() const { return static_cast<int>(threadIdx.x) % kAcross * E; }

  struct Load {
    __amdgpu_buffer_rsrc_t w;
    int lines, limit;  // lines and columns inside
    int alone;         // lines from here on end inside a chunk that nothing may be read behind
  };
  // The memory of the next load; `at` moves on.  Behind the last step nothing is inside.
  __device__ __forceinline__ Load next() {
    const int inside = max(0, min(left, KT));
    // Columns behind the rows of the tile meet no output that is stored: where a line follows in memory, the chunk
    // that goes over a line's end is read as a whole.
    const bool follows = !KC && !VEC && left > KT && line >= 16;
    const uint32_t bytes = KC ? full : full - static_cast<uint32_t>(KT - inside) * line + (follows ? 16 : 0);
    const Load l{window(at, left > 0 ? bytes : 0), KC ? rows : inside, KC ? left : rows,
                 KC || line < 16 ? 0 : follows ? KT : inside - 1};
    if (KC) full -= kSpan * KT * kSrc;
    at += ahead;
    left -= kSpan * KT;
    return l;
  }

  // Chunk j of a load: into registers, then into LDS.
  __device__ __forceinline__ void load(const Load& l, int j, Words& words) const {
    const int col = col_of();
    const uint32_t down = static_cast<uint32_t>(j * kLines) * line;
    if constexpr (VEC) {
      const uint32_t o = (KC && col >= l.limit ? kNowhere : off) + down;
      const u32x4 v = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(l.w, o, 0, 0));
#pragma unroll
      for (int e = 0; e < 4; ++e) words[j][e] = v[e];
    } else {
      // Whole chunks at the alignment of an element, which the memory instructions take; the one that goes over the
      // end of a line by elements, if nothing may be read there or (along k) it has to be zero.
      const bool in_line = line_of(j) < l.lines, alone = line_of(j) >= l.alone;
      const bool split = col < l.limit && col + E > l.limit && alone;
      const uint32_t o = off + down;
      const u32x4 v = __builtin_bit_cast(
          u32x4, __builtin_amdgcn_raw_buffer_load_b128(l.w, in_line && col < l.limit && !split ? o : kNowhere, 0, 0));
#pragma unroll
      for (int e = 0; e < 4; ++e) words[j][e] = v[e];
      if (in_line && split) {
        uint32_t e[E], here = o;
        asm volatile("" : "+v"(here));  // the elements' offsets are made here, not kept in registers through the loop
#pragma unroll
        for (int q = 0; q < E; ++q) {
          const uint32_t at_q = col + q < l.limit ? here + q * kSrc : kNowhere;
          if constexpr (ST == GASLOC_BF16)
            e[q] = static_cast<uint16_t>(__builtin_amdgcn_raw_buffer_load_b16(l.w, at_q, 0, 0));
          else
            e[q] = __builtin_amdgcn_raw_buffer_load_b32(l.w, at_q, 0, 0);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q)
          words[j][q] = ST == GASLOC_BF16 ? e[2 * q % E] | e[(2 * q + 1) % E] << 16 : e[q % E];
      }
    }
  }
  // Where chunk 0 of this thread goes, and the lane's part of the fragment that begins at row `row` of the tile.
  __device__ __forceinline__ uint32_t store_at(uint32_t lds) const {
    const int l = line_of(0), byte = col_of() * kSize;
    if constexpr (KC)
      return lds + byte / 64 * kLds + l * kStride + (byte % 64 / 16 ^ (0 - l / 4 & 3)) * 16 + byte % 16;
    else if constexpr (CT == GASLOC_BF16)
      return lds + l * kStride + (byte / 32 ^ across(l)) * 32 + byte % 32;
    else
      return lds + l * kStride + byte;
  }
  __device__ __forceinline__ static uint32_t read_at(uint32_t lds, int row) {
    const int l = lane_id(), i = l % 16, g = l / 16;
    if constexpr (KC)
      return lds + (row + i) * kStride + (g ^ (0 - i / 4 & 3)) * 16;
    else if constexpr (CT == GASLOC_BF16)
      return lds + (g * 8 + i / 4) * kStride + (row / 16 ^ across(g * 8 + i / 4)) * 32 + i % 4 * 8;
    else
      return lds + g * 4 * kStride + (row + i) * 4;
  }
  // How the 32-byte blocks of line k are permuted (of a line of 64 rows there are four).
  __device__ __forceinline__ static int across(int k) {
    return ROWS == 64 ? k % 4 ^ k / 8 % 2 : k % 4 + k / 8 % 2 * 4;
  }

  __device__ __forceinline__ void store(uint32_t to, int j, const Words& words) const {
    static_assert(!KC || kLines % 16 == 0, "a thread's rows are permuted alike");
    static_assert(KC || CT != GASLOC_BF16 || kLines % 8 == 0, "or by turns");
    // line k + 8 has its blocks exchanged by fours
    static_assert(KC || CT != GASLOC_BF16 || ROWS >= 128 || kLines % 16 == 0, "lines of 128 bytes stay as they are");
    if (!KC && CT == GASLOC_BF16 && kLines * j / 8 % 2 == 1) to ^= 128;
    to += j * kLines * kStride;
    if constexpr (ST == CT) {
      *lds_pointer<u32x4>(to) = u32x4{words[j][0], words[j][1], words[j][2], words[j][3]};
    } else {
      *lds_pointer<u32x2>(to) = u32x2{f32x2_to_bf16x2(__uint_as_float(words[j][0]), __uint_as_float(words[j][1])),
                                      f32x2_to_bf16x2(__uint_as_float(words[j][2]), __uint_as_float(words[j][3]))};
    }
  }
  // The fragment of sixteen rows, the p-th from the row `from` was made for: lane l has row l % 16, elements
  // E (l / 16) .. of the step's k.  `buffer`: how far the step's buffer lies behind the first.
  __device__ __forceinline__ static u32x4 fragment(uint32_t from, int buffer, int p) {
    if constexpr (KC) {
      return *lds_pointer<const u32x4>(from + buffer + p * 16 * kStride);
    } else if constexpr (CT == GASLOC_BF16) {
      // 16 lanes read four lines of k, 16 columns each; lane i gets column i
      const uint32_t at = (from ^ p % 8 * 32) + p / 8 * 256 + buffer;
      const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(lds_pointer<s16x4>(at)));
      const u32x2 hi =
          __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(lds_pointer<s16x4>(at + 4 * kStride)));
      return u32x4{lo.x, lo.y, hi.x, hi.y};
    } else {
      u32x4 v;
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = *lds_pointer<const uint32_t>(from + buffer + q * kStride + p * 64);
      return v;
    }
  }
};

template <int CT>
__device__ __forceinline__ f32x4 multiply(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (CT == GASLOC_BF16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                   0, 0);
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q)
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[q]), __uint_as_float(b[q]), c, 0, 0, 0);
    return c;
  }
}

// A tile of TM x TN outputs by WAVES_M x WAVES_N waves.  SPLIT: a workgroup takes `chunk` of k, and where a worker
// has several such parts it leaves its sums in `partial` for the join.
template <int PASS, int PT, int AT, int TM, int TN, int WAVES_M, int WAVES_N, bool VEC, bool SPLIT>
__global__ __launch_bounds__(kWave* WAVES_M* WAVES_N, 2) void k_linear(LinearArgs a) {
  constexpr int THREADS = kWave * WAVES_M * WAVES_N;
  constexpr bool kForward = PASS == kLinearForward, kWeight = PASS == kLinearWeight;
  using OpA = Operand<TM, THREADS, !kWeight, AT, AT, VEC>;
  using OpB = Operand<TN, THREADS, kForward, kWeight ? AT : PT, AT, VEC>;
  constexpr int KT = OpA::KT;
  constexpr int WM = TM / WAVES_M, WN = TN / WAVES_N, FM = WM / 16, FN = WN / 16;
  __shared__ __align__(16) char s_tiles[kBuffers * (OpA::kLds + OpB::kLds)];
  const uint32_t lds_a = static_cast<uint32_t>(
      reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)s_tiles));
  const uint32_t lds_b = lds_a + kBuffers * OpA::kLds;

  // Workgroups go round the eight XCDs.  Each XCD gets a contiguous stretch of tiles, which share rows of A or B in
  // its L2: of all the tiles, where tiles cost the same; of every worker's tiles in the weight's gradient, whose
  // cost is the worker's number of rows (the workers with the most rows come first, in `order`).
  const int b = blockIdx.x;
  const int owner = kWeight ? find_worker(a.tiles, a.n, b) : 0;
  const int from = kWeight ? a.tiles.begin[owner] : 0;
  const int total = a.tiles.begin[kWeight ? owner + 1 : a.n] - from;
  const int xcd = (b - from) % 8, each = total / 8, more = total % 8;
  const int t = from + xcd * each + (xcd < more ? xcd : more) + (b - from) / 8;
  const int span = kWeight ? owner : find_worker(a.tiles, a.n, t);
  const int i = kWeight ? a.order[span] : span;
  const int64_t r0 = a.rows.begin[i];
  const int count = a.rows.begin[i + 1] - a.rows.begin[i];
  const int M = kWeight ? a.out_features : count;
  const int N = kForward ? a.out_features : a.in_features;
  const int whole = kForward ? a.in_features : kWeight ? count : a.out_features;
  const int across = (N + TN - 1) / TN;
  // parts of k: first all tiles of the first part
  const int tiles = across * ((M + TM - 1) / TM);
  const int part = SPLIT ? (t - a.tiles.begin[span]) / tiles : 0;
  const int tile = t - a.tiles.begin[span] - part * tiles;
  const int k_first = SPLIT ? part * a.chunk : 0;
  const int depth = SPLIT ? min(whole - k_first, a.chunk) : whole;
  // kGroup tiles of m by all of n at a time, m first: the tiles that an XCD works on at once are about as many of m as
  // of n, which is what has to be read least for.
  constexpr int kGroup = TM == 256 ? 4 : 8;
  const int group = tile / (kGroup * across), in_group = tile % (kGroup * across);
  const int tall = min(kGroup, (M + TM - 1) / TM - group * kGroup);
  const int m0 = (group * kGroup + in_group % tall) * TM, n0 = in_group / tall * TN;
  constexpr int kAct = AT == GASLOC_BF16 ? 2 : 4, kPar = PT == GASLOC_BF16 ? 2 : 4;
  const char* w = static_cast<const char*>(live_row<PT>(a.w, i)) + a.weight * kPar;

  OpA oa;
  OpB ob;
  if constexpr (kForward) {
    oa.start(static_cast<const char*>(a.x) + ((r0 + m0) * a.x_ld + k_first) * kAct, a.x_ld, M - m0, depth);
    ob.start(w + (static_cast<int64_t>(n0) * whole + k_first) * kPar, whole, N - n0, depth);
  } else if constexpr (!kWeight) {
    oa.start(static_cast<const char*>(a.dout) + ((r0 + m0) * a.dout_ld + k_first) * kAct, a.dout_ld, M - m0, depth);
    ob.start(w + (static_cast<int64_t>(k_first) * N + n0) * kPar, N, N - n0, depth);
  } else {
    oa.start(static_cast<const char*>(a.dout) + ((r0 + k_first) * a.dout_ld + m0) * kAct, a.dout_ld, M - m0, depth);
    ob.start(static_cast<const char*>(a.x) + ((r0 + k_first) * a.x_ld + n0) * kAct, a.x_ld, N - n0, depth);
  }

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int wm = wave / WAVES_N * WM, wn = wave % WAVES_N * WN;
  f32x4 c[FM][FN];
#pragma unroll
  for (int p = 0; p < FM; ++p) {
#pragma unroll
    for (int q = 0; q < FN; ++q) c[p][q] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }

  if (depth > 0) {
    // In step k its fragments are multiplied, those of step k + 1 are read from the next buffer, step k + 2 (and k + 3,
    // of an operand that is loaded two steps at a time, in even steps) is stored into the buffers after it, and what
    // follows is loaded: all of it in between the rows of products, so that the matrix cores do not wait for any of
    // it.  Behind the last step loads give zeros: there is no branch in the loop.
    constexpr int CA = OpA::kChunks, CB = OpB::kChunks;
    const uint32_t put_a = oa.store_at(lds_a), put_b = ob.store_at(lds_b);
    const uint32_t get_a = OpA::read_at(lds_a, wm), get_b = OpB::read_at(lds_b, wn);
    typename OpA::Words wa;
    typename OpB::Words wb;
    {
      typename OpA::Words wa0, wa1;
      typename OpB::Words wb0, wb1;
      const auto load_a = [&](typename OpA::Words& to) {
        const auto l = oa.next();
#pragma unroll
        for (int j = 0; j < CA; ++j) oa.load(l, j, to);
      };
      const auto load_b = [&](typename OpB::Words& to) {
        const auto l = ob.next();
#pragma unroll
        for (int j = 0; j < CB; ++j) ob.load(l, j, to);
      };
      load_a(wa0);
      load_b(wb0);
      if (OpA::kSpan == 1) load_a(wa1);
      if (OpB::kSpan == 1) load_b(wb1);
      load_a(wa);
      load_b(wb);
#pragma unroll
      for (int j = 0; j < CA; ++j) oa.store(put_a, j, wa0);
#pragma unroll
      for (int j = 0; j < CB; ++j) ob.store(put_b, j, wb0);
      if (OpA::kSpan == 1) {
#pragma unroll
        for (int j = 0; j < CA; ++j) oa.store(put_a + OpA::kLds, j, wa1);
      }
      if (OpB::kSpan == 1) {
#pragma unroll
        for (int j = 0; j < CB; ++j) ob.store(put_b + OpB::kLds, j, wb1);
      }
    }
    __syncthreads();
    u32x4 fa[4], fb[2][FN];  // A's fragments are read four rows ahead
    static_assert(FM % 4 == 0, "the rows go round the fragments evenly");
#pragma unroll
    for (int p = 0; p < 4; ++p) fa[p] = OpA::fragment(get_a, 0, p);
#pragma unroll
    for (int q = 0; q < FN; ++q) fb[0][q] = OpB::fragment(get_b, 0, q);
#pragma unroll 1
    for (int k0 = 0; k0 < depth; k0 += kBuffers * KT) {
#pragma unroll
      for (int cur = 0; cur < kBuffers; ++cur) {
        constexpr int kMask = kBuffers - 1;
        const int next = cur + 1 & kMask, free = cur + 2 & kMask, h = cur & 1;
        const bool do_a = OpA::kSpan == 1 || h == 0, do_b = OpB::kSpan == 1 || h == 0;
        typename OpA::Load la;
        typename OpB::Load lb;
        if (do_a) la = oa.next();
        if (do_b) lb = ob.next();
#pragma unroll
        for (int p = 0; p < FM; ++p) {
#pragma unroll
          for (int q = 0; q < FN; ++q) c[p][q] = multiply<AT>(fb[h][q], fa[p % 4], c[p][q]);  // lane: row l % 16 of C
          fa[p % 4] = p + 4 < FM ? OpA::fragment(get_a, cur * OpA::kLds, p + 4)
                                 : OpA::fragment(get_a, next * OpA::kLds, p + 4 - FM);
#pragma unroll
          for (int q = p * FN / FM; q < (p + 1) * FN / FM; ++q)
            fb[h ^ 1][q] = OpB::fragment(get_b, next * OpB::kLds, q);
#pragma unroll
          for (int j = p * CA / FM; j < (p + 1) * CA / FM && do_a; ++j) {
            oa.store(put_a + free * OpA::kLds, j, wa);
            oa.load(la, j, wa);
          }
#pragma unroll
          for (int j = p * CB / FM; j < (p + 1) * CB / FM && do_b; ++j) {
            ob.store(put_b + free * OpB::kLds, j, wb);
            ob.load(lb, j, wb);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
        __syncthreads();
      }
    }
  }

  // Lane l holds row l % 16 and columns 4 (l / 16) .. + 3 of each 16 x 16 block.  Sixteen rows at a time go
  // through the wave's own part of LDS, so that whole lines are stored.
  using Out = typename std::conditional<kWeight || AT == GASLOC_F32 || SPLIT, float, uint16_t>::type;
  constexpr int kOutStride = WN * static_cast<int>(sizeof(Out)) + 16;
  constexpr int V = 16 / static_cast<int>(sizeof(Out));
  static_assert(THREADS / kWave * 16 * kOutStride <= kBuffers * (OpA::kLds + OpB::kLds),
                "sixteen rows of every wave fit");
  char* const mine = s_tiles + wave * 16 * kOutStride;
  const int lane = lane_id();
  Out* out;
  int64_t out_ld = kWeight ? N : a.out_ld;
  const bool split = SPLIT && a.parts.begin[span + 1] - a.parts.begin[span] > 1;
  bool add = false;
  if (split) {
    // weight: one matrix per part of every worker; else one set of all rows per part
    const int64_t at = kWeight ? static_cast<int64_t>(a.parts.begin[span] + part) * M * N
                               : (static_cast<int64_t>(part) * a.rows.begin[a.n] + r0) * N;
    out = reinterpret_cast<Out*>(a.partial + at);
    out_ld = N;
  } else if constexpr (kWeight) {
    out = a.grads + static_cast<int64_t>(i) * a.grad_ld + a.weight;
    add = a.accumulate;
  } else {
    out = static_cast<Out*>(a.out) + r0 * a.out_ld;
  }
#pragma unroll
  for (int p = 0; p < FM; ++p) {
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int q = 0; q < FN; ++q) {
      char* to = mine + lane % 16 * kOutStride + (16 * q + lane / 16 * 4) * static_cast<int>(sizeof(Out));
      if constexpr (sizeof(Out) == 4)
        *reinterpret_cast<f32x4*>(to) = c[p][q];
      else
        *reinterpret_cast<u32x2*>(to) =
            u32x2{f32x2_to_bf16x2(c[p][q][0], c[p][q][1]), f32x2_to_bf16x2(c[p][q][2], c[p][q][3])};
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const int top = m0 + wm + 16 * p;
#pragma unroll 4
    for (int e = lane * V; e < 16 * WN; e += kWave * V) {
      const int row = e / WN, col = e % WN, n = n0 + wn + col;
      if (top + row >= M || n >= N) continue;
      const char* from = mine + row * kOutStride + col * static_cast<int>(sizeof(Out));
      Out* to = out + (top + row) * out_ld + n;
      if constexpr (VEC && kWeight) {
        f32x4 v = *reinterpret_cast<const f32x4*>(from);
        if (add) v += *reinterpret_cast<const f32x4*>(to);
        *reinterpret_cast<f32x4*>(to) = v;
      } else if constexpr (VEC) {
        *reinterpret_cast<u32x4*>(to) = *reinterpret_cast<const u32x4*>(from);
      } else if (n + V <= N) {  // at the alignment of an element
        u32x4 v = *reinterpret_cast<const u32x4*>(from);
        if constexpr (kWeight) {
          if (add) v = __builtin_bit_cast(u32x4, __builtin_bit_cast(f32x4, load_words4<false>(to)) +
                                                     __builtin_bit_cast(f32x4, v));
        }
        *reinterpret_cast<u32x4_any*>(to) = v;
      } else {
#pragma unroll
        for (int q = 0; q < V; ++q) {
          if (n + q < N) {
            const Out v = reinterpret_cast<const Out*>(from)[q];
            if constexpr (kWeight)
              to[q] = add ? to[q] + v : v;
            else
              to[q] = v;
          }
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

// Adds the parts of a split product in order and stores the sums: for the weight's gradient those of the worker of
// span blockIdx.y (if it has more than one part), else all rows.
template <int PASS, int AT>
__global__ __launch_bounds__(256) void k_linear_join(LinearArgs a) {
  constexpr bool kWeight = PASS == kLinearWeight;
  const int span = blockIdx.y;
  const int parts = a.parts.begin[span + 1] - a.parts.begin[span];
  if (kWeight && parts < 2) return;
  const int N = PASS == kLinearForward ? a.out_features : a.in_features;
  const int64_t all = static_cast<int64_t>(kWeight ? a.out_features : a.rows.begin[a.n]) * N;
  const float* p = a.partial + (kWeight ? a.parts.begin[span] * all : 0);
  for (int64_t e = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; e < all; e += gridDim.x * 256ll) {
    float sum = p[e];
#pragma unroll 4
    for (int k = 1; k < parts; ++k) sum += p[k * all + e];
    if constexpr (kWeight) {
      float* to = a.grads + static_cast<int64_t>(a.order[span]) * a.grad_ld + a.weight + e;
      *to = a.accumulate ? *to + sum : sum;
    } else {
      const int64_t at = e / N * a.out_ld + e % N;
      if constexpr (AT == GASLOC_BF16)
        static_cast<uint16_t*>(a.out)[at] = static_cast<uint16_t>(f32x2_to_bf16x2(sum, 0.0f) & 0xffffu);
      else
        static_cast<float*>(a.out)[at] = sum;
    }
  }
}

// Forward pass of workers with at most kFewRows rows each: reading the weights is all there is to it, so they go from
// memory to the matrix cores through registers, 16 outputs per workgroup, each of its four waves a quarter of k.
// Lane l has output l % 16 of the weights and row l % 16 of x.  bf16 weights: of every 32 of k the 8 from 8 (l / 16)
// on; fp32 ones: the 4 from 4 (l / 16) on and the 4 that lie 16 behind them.  Either way a load takes 64 bytes of 16
// rows, and the other half of those lines is next, so the loads go through the caches (streaming ones took 52 us).
// Bound by HBM: one row of n = 16, 2048 -> 2048, fp32 weights 46 to 48 us (5.6 to 5.8 TB/s), bf16 weights 28 (4.9).
// More rows take longer, 4 each 52 us and 16 each 71, where tiles of 64 take 62 (17 rows each).
template <int PT, int AT>
__global__ __launch_bounds__(256) void k_linear_rows(LinearArgs a) {
  constexpr int kAhead = 4;                        // 32s of k in flight
  constexpr int V = PT == GASLOC_BF16 ? 8 : 4;     // of k per load
  constexpr int H = 8 / V;
  __shared__ f32x4 s_sum[4][kWave];
  const int i = find_worker(a.tiles, a.n, blockIdx.x);
  const int64_t r0 = a.rows.begin[i];
  const int rows = a.rows.begin[i + 1] - a.rows.begin[i];
  const int N = a.out_features, K = a.in_features;
  const int n0 = (static_cast<int>(blockIdx.x) - a.tiles.begin[i]) * 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = lane_id();
  const int quarter = (K + 4 * 32 - 1) / (4 * 32) * 32;
  const int k_first = wave * quarter, k_end = min(K, k_first + quarter);
  const int mine = n0 + lane % 16;
  const int64_t w_at = a.weight + static_cast<int64_t>(mine < N ? mine : N - 1) * K;
  const int64_t x_at = (r0 + (lane % 16 < rows ? lane % 16 : 0)) * a.x_ld;
  const bool has_row = lane % 16 < rows;
  const void* w = live_row<PT>(a.w, i);
  f32x4 c = {0.0f, 0.0f, 0.0f, 0.0f};
  // WHOLE: all of the block lies inside, so that its loads are issued back to back
  const auto block = [&](int k_block, auto whole) {
    constexpr bool kWhole = decltype(whole)::value;
    constexpr int kDeep = kWhole ? kAhead : 1;
    float fw[kDeep][8], fx[kDeep][8];
#pragma unroll
    for (int q = 0; q < kDeep; ++q) {
#pragma unroll
      for (int h = 0; h < H; ++h) {
        const int k = k_block + lane / 16 * V + 32 * q + 16 * h, left = kWhole ? V : max(0, k_end - k);
        float pw[V], px[V];
        load_row<PT, V, false>(w, w_at + k, left, pw);
        load_row<AT, V, false>(a.x, x_at + k, left, px);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          fw[q][h * V + e] = pw[e];
          fx[q][h * V + e] = px[e];
        }
      }
    }
    if (kWhole) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int q = 0; q < kDeep; ++q) {
#pragma unroll
      for (int e = 0; e < 8; ++e) fx[q][e] = has_row ? fx[q][e] : 0.0f;
      if constexpr (AT == GASLOC_BF16) {
        u32x4 fa, fb;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          fa[e] = f32x2_to_bf16x2(fw[q][2 * e], fw[q][2 * e + 1]);
          fb[e] = f32x2_to_bf16x2(fx[q][2 * e], fx[q][2 * e + 1]);
        }
        c = multiply<AT>(fa, fb, c);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(fw[q][e], fx[q][e], c, 0, 0, 0);
      }
    }
  };
  int k = k_first;
  for (; k + 32 * kAhead <= k_end; k += 32 * kAhead) block(k, std::true_type{});
  for (; k < k_end; k += 32) block(k, std::false_type{});
  s_sum[wave][lane] = c;
  __syncthreads();
  if (wave != 0 || !has_row) return;
#pragma unroll
  for (int k = 1; k < 4; ++k) c += s_sum[k][lane];
  // the lane holds outputs n0 + 4 (l / 16) .. + 3 of row l % 16
  const int n = n0 + lane / 16 * 4;
  const float o[4] = {c[0], c[1], c[2], c[3]};
  if (n < N) store_row<AT, 4>(a.out, (r0 + lane % 16) * a.out_ld + n, N - n, o);
}

// Tiles of four waves, whose sums may be split.
template <int PASS, int PT, int AT, int TILE, int WAVES_M, int WAVES_N>
hipError_t launch_small(const LinearArgs& a, bool vec, hipStream_t stream) {
  const bool split = a.chunk != 0;
  return launch_kernel(vec ? split ? k_linear<PASS, PT, AT, TILE, TILE, WAVES_M, WAVES_N, true, true>
                                   : k_linear<PASS, PT, AT, TILE, TILE, WAVES_M, WAVES_N, true, false>
                       : split ? k_linear<PASS, PT, AT, TILE, TILE, WAVES_M, WAVES_N, false, true>
                               : k_linear<PASS, PT, AT, TILE, TILE, WAVES_M, WAVES_N, false, false>,
                       dim3(a.tiles.begin[a.n]), 256, 0, stream, a);
}

template <int PASS, int PT, int AT>
hipError_t launch_types(const LinearArgs& a, int tile, bool vec, hipStream_t stream) {
  const dim3 grid(a.tiles.begin[a.n]);
  if constexpr (AT == GASLOC_BF16) {
    if (tile == 256)
      return launch_kernel(k_linear<PASS, PT, AT, 256, 256, 2, 4, true, false>, grid, 512, 0, stream, a);
  }
  if constexpr (PASS == kLinearForward) {
    if (tile == kFewRows) return launch_kernel(k_linear_rows<PT, AT>, grid, 256, 0, stream, a);
  }
  const hipError_t e = tile == 64 ? launch_small<PASS, PT, AT, 64, 1, 4>(a, vec, stream)
                                  : launch_small<PASS, PT, AT, 128, 2, 2>(a, vec, stream);
  if (e != hipSuccess || a.chunk == 0) return e;
  const int N = PASS == kLinearForward ? a.out_features : a.in_features;
  const int64_t all = static_cast<int64_t>(PASS == kLinearWeight ? a.out_features : a.rows.begin[a.n]) * N;
  const dim3 join(static_cast<unsigned>(all / 256 < 2048 ? (all + 255) / 256 : 2048), PASS == kLinearWeight ? a.n : 1);
  return launch_kernel(k_linear_join<PASS, AT>, join, 256, 0, stream, a);
}

template <int PASS>
hipError_t launch(const LinearArgs& a, int params, int act, int tile, bool vec, hipStream_t stream) {
  // the weight's gradient does not read the parameters
  if (PASS != kLinearWeight && params == GASLOC_BF16)
    return launch_types<PASS, PASS == kLinearWeight ? GASLOC_F32 : GASLOC_BF16, GASLOC_BF16>(a, tile, vec, stream);
  if (act == GASLOC_BF16) return launch_types<PASS, GASLOC_F32, GASLOC_BF16>(a, tile, vec, stream);
  return launch_types<PASS, GASLOC_F32, GASLOC_F32>(a, tile, vec, stream);
}

}  // namespace

hipError_t launch_linear(const LinearArgs& a, LinearPass pass, int params, int act, int tile, bool vec,
                         hipStream_t stream) {
  if (pass == kLinearForward) return launch<kLinearForward>(a, params, act, tile, vec, stream);
  if (pass == kLinearInput) return launch<kLinearInput>(a, params, act, tile, vec, stream);
  return launch<kLinearWeight>(a, params, act, tile, vec, stream);
}

}  // namespace gasloc
