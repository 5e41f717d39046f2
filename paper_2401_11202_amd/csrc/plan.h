// Plans and their execution: what the host side of every entry point builds
// (a list of kernel launches), and the steps they share -- the thread-local
// error message, the plan's text, the workspace check and the enqueue.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdlib>
#include <functional>
#include <memory>
#include <string>
#include <utility>
#include <vector>

#include "../../include/partir.h"
#include "kernels.h"

namespace partir {

constexpr int kNumCU = 256;           // MI355X compute units: a grid below this underfills
constexpr size_t kWsAlign = 256;

extern thread_local std::function<void()> g_deferred_text;   // builds the text of the last call's plan, if it is wanted

// Whether the plan being built on this thread needs its text: formatting takes
// as long as planning, and only partir_last_plan_text reads what a call that
// executes would leave.
extern thread_local bool g_want_text;

struct TextScope {
  explicit TextScope(bool want) { g_want_text = want; }
  ~TextScope() { g_want_text = true; }
};

// snprintf into a plan's text; empty when no text is wanted
void textf(char* buf, size_t n, const char* fmt, ...);
// Records the thread's error message and returns the status.
int fail(int status, const char* fmt, ...);

inline size_t align_up(size_t x) { return (x + kWsAlign - 1) / kWsAlign * kWsAlign; }
inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// ---------------------------------------------------------------------------
// Plans
// ---------------------------------------------------------------------------
enum LaunchKind { L_GEMM_BF16, L_GEMM_F32, L_REDUCE, L_ATTN, L_ATTN_COMBINE, L_RMS, L_ACT_BWD, L_COLSUM,
                  L_GEMM_BF16_PARTS, L_ATTN_BWD, L_RMS_PARTS, L_GEMM_BF16_FIXUP, L_GEMM_BF16_PARTS_FIXUP, L_CALL };

struct Launch {
  LaunchKind kind;
  std::string name;
  std::string text;
  GemmParams gemm{};
  GemmF32Params gemm32{};
  ReduceParams reduce{};
  AttnParams attn{};
  RmsParams rms{};
  ActBwdParams act{};
  ColSumParams cs{};
  std::shared_ptr<GemmParts> parts;   // L_GEMM_BF16_PARTS: the device-local arrays
  std::shared_ptr<RmsParts> rms_parts;   // L_RMS_PARTS
  AttnBwdParams attn_bwd{};
  std::function<hipError_t(hipStream_t)> call;   // L_CALL: enqueues one kernel
};

struct Plan {
  std::vector<Launch> launches;
  int n_shards = 1;
  int n_tile_loops = 0;
  int n_sum_loops = 0;
  int n_sum_splitk = 0;
  size_t ws_bytes = 0;
  double flops = 0;
};

// ---------------------------------------------------------------------------
// Execution
// ---------------------------------------------------------------------------
void keep_plan_text(const Plan& plan, const char* what);
void fill_info(const Plan& plan, partir_plan_info* info);
int check_ws(const Plan& plan, void* ws, size_t ws_bytes);
// A pointer the plan depends on only by being there: its text is planned again
// later with a stand-in, so that no caller's pointer outlives the call.
template <typename T>
void stand_in(T*& p) {
  if (p) p = (T*)(uintptr_t)kWsAlign;
}

int execute(const Plan& plan, void* stream);

// A call that executes: plans it once (with its workspace), runs it, and
// leaves the text to partir_last_plan_text.
template <typename Args>
int run_plan(const char* what, const Args& a, void (*planner)(const Args&, void*, Plan&), void* ws, size_t ws_bytes,
             void* stream) {
  const char* dump = getenv("PARTIR_DUMP_PLAN");
  const bool now = dump && dump[0] == '1';
  Plan plan;
  plan.launches.reserve(12);
  {
    TextScope scope(now);
    planner(a, ws, plan);
  }
  const int st = check_ws(plan, ws, ws_bytes);
  if (st) return st;
  if (now) {
    keep_plan_text(plan, what);
  } else {
    Args sizes = a;
    sizes.drop_pointers();
    g_deferred_text = [what, sizes, planner] {
      Plan again;
      planner(sizes, nullptr, again);
      keep_plan_text(again, what);
    };
  }
  return execute(plan, stream);
}

}  // namespace partir
