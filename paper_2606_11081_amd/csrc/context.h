// A context and what every C entry point of it shares (runtime.cpp, layers.cpp):
// error records, the device guard, small argument checks.  Not installed.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstdint>
#include <string>
#include <vector>

#include "gasloc.h"
#include "internal.h"

namespace gasloc {
constexpr int kStageSlots = 4;  // pinned CSR staging slots, reused round-robin
}

struct gasloc_ctx {
  int n = 0;
  int64_t P = 0;
  gasloc_topology topo{};
  gasloc_hparams hp{};
  gasloc_buffers buf{};
  hipStream_t stream = nullptr;
  int device = 0;
  int cus = 0;

  std::vector<uint8_t> admissible;  // copy of the topology's admissible graph (or empty)
  std::vector<uint8_t> alive;       // 1 per live worker
  bool any_dead = false;
  std::vector<int32_t> skip_rp, skip_col;  // scratch for skipped exchanges
  std::vector<float> skip_val;
  std::vector<int32_t> plan_ops;  // visit plan of the current round
  std::vector<int64_t> k;         // AdamW step count per worker
  std::vector<uint8_t> stepped;   // local steps taken since the last round
  int64_t rounds_done = 0;
  bool ce_current = false;        // h_stats[0] is (or will be, in stream order) the consensus error of the stored x
  bool failed = false;

  unsigned char* d_csr = nullptr;  // device copy of the round's CSR or visit plan
  std::vector<unsigned char> d_csr_key;  // what d_csr holds (kind byte + contents), to skip repeats
  unsigned char* h_stage[gasloc::kStageSlots] = {};
  hipEvent_t stage_done[gasloc::kStageSlots] = {};
  bool stage_used[gasloc::kStageSlots] = {};
  int stage_next = 0;
  // [kPartialWords]: consensus-error partials, pseudo-gradient partials (each
  // kMaxPartials), then the finalize's segment sums
  double* d_partials = nullptr;
  // [2]: consensus error, squared pseudo-gradients of the last round, in pinned
  // host memory that the finalize kernel writes (d_stats: its device address);
  // a reader waits for the stream and reads the host side
  double* h_stats = nullptr;
  double* d_stats = nullptr;

  size_t lds_per_block_max = 0;
  size_t lds_per_cu = 0;

  std::string err;
  // scratch for generated CSRs
  std::vector<int32_t> row_ptr, col;
  std::vector<float> val;
};

namespace gasloc {

std::string format(const char* fmt, ...);
// Record the message of a failing call (on the thread without a context); a device error makes
// the context unusable.
gasloc_status fail(gasloc_ctx* ctx, gasloc_status st, const std::string& msg);
gasloc_status hip_fail(gasloc_ctx* ctx, hipError_t e, const char* what);

#define HIP_TRY(ctx, call)                                   \
  do {                                                       \
    hipError_t e_ = (call);                                  \
    if (e_ != hipSuccess) return gasloc::hip_fail((ctx), e_, #call); \
  } while (0)

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline size_t param_bytes(int dtype) { return dtype == GASLOC_BF16 ? 2 : 4; }

// Makes ctx->device current for the duration of an ABI call.
class DeviceGuard {
 public:
  explicit DeviceGuard(int device) {
    if (hipGetDevice(&prev_) == hipSuccess && prev_ != device) {
      if (hipSetDevice(device) == hipSuccess) restore_ = true;
    }
  }
  ~DeviceGuard() {
    if (restore_) (void)hipSetDevice(prev_);
  }

 private:
  int prev_ = -1;
  bool restore_ = false;
};

}  // namespace gasloc
