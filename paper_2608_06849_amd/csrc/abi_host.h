// Argument checks and the head-scheduling pass (abi.cpp), for the units that hold
// entry points of aoh.h.
#pragma once
#include <stdint.h>

#include "aoh.h"
#include "aoh_internal.h"

namespace aoh {

// Sets the thread's last-error text and returns the status / clears it.
aoh_status fail(aoh_status st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
aoh_status ok();

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

int compute_units();

aoh_status check_tensor(const aoh_tensor* t, const char* name, int ndim, int dtype_a, int dtype_b);
aoh_status check_mask_params(int n_sink, int window);
aoh_status check_paged(const aoh_paged_cache* c, int n_ret, int64_t B);
aoh_status check_ring(const aoh_ring_cache* c, int n_str, int n_sink, int window, int64_t B);

// Head-scheduling pass: KV-head lists by label (ascending id) and each KV
// head's rank inside its cache.
struct HeadSchedule {
  int n_ret = 0, n_str = 0;
  uint8_t ret[kMaxKvHeads];
  uint8_t str[kMaxKvHeads];
  uint8_t rank[kMaxKvHeads];
  uint64_t streaming_mask = 0;
};

aoh_status schedule_heads(const uint8_t* head_is_streaming, int hkv, HeadSchedule* hs);

}  // namespace aoh
