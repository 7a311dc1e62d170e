// The pool handle and the host helpers that its entry points share
// (gambit_pool.cpp: bookkeeping, decode steps, thought boundaries;
// rows_attn.cpp: packed writes, prompt and draft-tree attention).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <string>
#include <vector>

#include "../../include/gambit.h"
#include "kernels.h"
#include "rows.h"

namespace gambit {
namespace host {

constexpr size_t kAlign = 256;
constexpr int kDefaultSplits = 64;
constexpr int kMaxLayers = 1024;

inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
inline int cdiv(int a, int b) { return (a + b - 1) / b; }

// Workspace carve-up.  All offsets are kAlign-aligned.
struct Layout {
  size_t list, ids, req_trace, req_ntok, pairs, free_list, nk, ticket, queues, err, scales, freebits,
      alloc_list, units, members, part_ml, part_acc, sbar, nscore, gen, ghost, tourn, rows_plan[2], write_plan, total;
  int kmax, max_units, max_members, nwords;
  // packed tokens: most of one call, partials (Hq rows each) of a rows plan;
  // the items of a plan of prompts and of one of trees, and their bytes
  int max_packed, max_parts, max_items[2];
  size_t rows_plan_bytes[2], write_plan_bytes;
};

// A plan of packed tokens kept for calls that list the same (the layers of a
// step): the mirror it was made from, and what the call listed.
struct PackedKey {
  bool valid = false;
  uint64_t epoch = 0;
  std::vector<int32_t> listed;
};

// The kept plan of one kind of call, and its pinned image, reused after `ev`.
// A kind each, so that a layer's write, prompt and tree calls keep theirs.
template <class Launch>
struct KeptPlan {
  PackedKey key;
  Launch launch{};
  uint8_t* image = nullptr;
  hipEvent_t ev = nullptr;
};
enum { kPromptPlan = 0, kTreePlan = 1 };

}  // namespace host
}  // namespace gambit

struct gambit_pool {
  gambit_pool_desc d{};
  gambit::host::Layout L{};
  gambit::DevPool dev{};
  uint8_t* ws = nullptr;
  int g = 1;
  int n_cu = 256;  // compute units of the pool's device (two attention workgroups each)
  float append_scale = 1.f / 64.f;

  // host mirror
  std::vector<std::vector<int32_t>> table;
  std::vector<int32_t> seq_len, refcount;
  // tournament bookkeeping (Alg. 1): scored thoughts, tokens generated since
  // creation, ghost flag; the scores themselves live on the device only
  std::vector<int32_t> nscore, gen;
  std::vector<char> ghost;
  std::vector<uint64_t> freebits;  // bit set = free
  int32_t nfree = 0;
  size_t hint = 0;                 // no free bit below word `hint`

  // pinned staging for host-to-device copies, reused after an event fence
  int32_t* stage = nullptr;
  size_t stage_ints = 0;
  hipEvent_t stage_ev = nullptr;
  uint8_t* plan_stage = nullptr;
  size_t plan_stage_bytes = 0;
  hipEvent_t plan_ev = nullptr;

  // attention plan
  bool plan_valid = false;
  std::vector<int32_t> plan_list;
  int xcd_off[9] = {0};
  int plan_steps = 0;              // decode steps taken with the plan
  size_t plan_partials = 0;        // partials of one head that a launch with the plan writes
  int grid = 0;
  int n_units = 0;
  bool queues_dirty = false;       // an attention launch was not followed by its merge
  int max_splits_used = 0;
  int step_next = 0;               // the layer the open decode step expects next (0: none open)
  gambit::AttnLaunch step{};       // the open step's launch arguments
  std::vector<int32_t> cnt, first;  // per-block planner scratch, zero / -1 between calls
  gambit_stats stats{};            // of plan_list, kept current by decode steps
  std::vector<int32_t> plan_kinds;  // per list position: GAMBIT_UNIT_* bits of the units covering it

  // packed tokens (rows_attn.cpp): the kept plans, their images one pinned
  // buffer; changes of the mirror's lengths or rows so far
  uint64_t epoch = 0;
  int device = 0;
  uint8_t* packed_stage = nullptr;
  gambit::host::KeptPlan<gambit::RowsLaunch> rows[2];
  gambit::host::KeptPlan<gambit::WriteLaunch> write;

  // attention-kernel event timing
  std::vector<hipEvent_t> prof_ev;
  int prof_used = 0;
  bool prof_on = false;

  std::string last_error;
};

namespace gambit {
namespace host {

inline gambit_status fail(gambit_pool* p, gambit_status s, const char* fmt, ...) {
  if (p) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    p->last_error = buf;
  }
  return s;
}

inline gambit_status hip_fail(gambit_pool* p, hipError_t e, const char* where) {
  return fail(p, GAMBIT_ERR_DEVICE, "%s: %s", where, hipGetErrorString(e));
}

#define HIP_TRY(p, expr, where)                 \
  do {                                          \
    const hipError_t e_ = (expr);               \
    if (e_ != hipSuccess) return hip_fail(p, e_, where); \
  } while (0)

inline hipStream_t S(void* s) { return static_cast<hipStream_t>(s); }

template <class T>
T* ws_ptr(gambit_pool* p, size_t off) {
  return reinterpret_cast<T*>(p->ws + off);
}

inline gambit_status check_ids(gambit_pool* p, int32_t n, const int32_t* ids, const char* what,
                        std::vector<char>* seen_out = nullptr) {
  if (n < 0 || n > p->d.max_traces) return fail(p, GAMBIT_ERR_INVALID, "%s count %d out of range", what, n);
  if (n > 0 && !ids) return fail(p, GAMBIT_ERR_INVALID, "%s list is NULL", what);
  std::vector<char> seen(p->d.max_traces, 0);
  for (int i = 0; i < n; ++i) {
    const int t = ids[i];
    if (t < 0 || t >= p->d.max_traces) return fail(p, GAMBIT_ERR_INVALID, "%s id %d out of range", what, t);
    if (seen[t]) return fail(p, GAMBIT_ERR_INVALID, "duplicate %s id %d", what, t);
    seen[t] = 1;
  }
  if (seen_out) seen_out->swap(seen);
  return GAMBIT_OK;
}

// Calls that change or check the pool wait for an open decode step to end.
inline gambit_status step_open(gambit_pool* p) {
  return fail(p, GAMBIT_ERR_INVALID, "a decode step is open: layer %d of %d is next", p->step_next,
              p->dev.num_layers);
}

}  // namespace host
}  // namespace gambit
