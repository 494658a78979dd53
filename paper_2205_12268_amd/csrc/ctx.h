// What a context holds, for the translation units that define entry points of the C ABI.
#pragma once

#include <hip/hip_runtime.h>

#include "wcc.h"

struct wcc_ctx {
  int device = 0;               // the device wcc_create was given: owner of static_ws
  void *static_ws = nullptr;    // that device's copy of `scratch`
  void *ws = nullptr;
  size_t ws_bytes = 0;
  bool profiling = false;
  bool have_times = false;
  hipEvent_t ev[WCC_T_COUNT][2] = {};
  bool ev_ok = false;
  bool marked[WCC_T_COUNT] = {};  // stage bracket recorded by the last profiled call
  int block_profile_layer = 1;  // which layer of wcc_block_forward the stage events bracket
};

#define WCC_TRY(expr)                                 \
  do {                                                \
    if ((expr) != hipSuccess) return WCC_ERR_HIP;     \
  } while (0)
