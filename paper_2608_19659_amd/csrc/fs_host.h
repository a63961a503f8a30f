// fs_host.h -- what the host files of libfleetsieve share: the context, the
// thread's last error, and the guard that makes a context's device current.
#pragma once

#include <cstdlib>
#include <string>
#include <vector>

#include <hip/hip_runtime.h>

#include "fleetsieve.h"

struct fs_context {
  int device;
  int score_kernel;  // 0 auto, 1 wave per scenario, 2 lane per scenario, 3 exclusion
  int timing;        // back-to-back scoring-kernel launches between timing events (0 = off)
  int spl;           // exclusion scorer samples per lane (0 = default)
  int waves;         // exclusion scorer grid in wavefronts (0 = default)
  int setup;         // exclusion scorer set-up: 0 automatic, 1 general
  int loop_objective;  // profiling loop certificate: 0 max-min, 1 whole objective
  int loop_refit;      // profiling loop fit step: 0 off, 1 interval refit every round
  int thr_search;      // exclusion set-up: capacity-threshold search start (0 window, 1 stepping, 2 bisection)
  int attention;       // cache attention: 0 by size, 1 the kernel of 16 rows, 2 that of 256
  int32_t *pinned;   // pinned host word: running trajectories read back by fs_profile_loop
  void *scratch;     // this device's address of the static scratch of fs_score_candidates_noalloc
  // a second stream (default priority) and the fork / join events of the
  // stage-wise score; the profiling loop waits on the fork event for its count
  hipStream_t side;
  hipEvent_t fork, join;
  struct Timed {
    hipEvent_t begin, end;
    int launches;
  };
  std::vector<Timed> events;
};

namespace fs {

inline thread_local std::string g_error;

inline fs_status fail(fs_status s, const std::string &msg) {
  g_error = msg;
  return s;
}

inline fs_status hip_fail(hipError_t e, const char *what) {
  return fail(FS_ERR_DEVICE, std::string(what) + ": " + hipGetErrorString(e));
}

inline bool env_validate() {
  const char *v = std::getenv("FS_VALIDATE");
  return v && v[0] == '1';
}

struct DeviceGuard {
  int prev = -1;  // device to restore (-1: none, already current)
  hipError_t err = hipSuccess;
  explicit DeviceGuard(int dev) {
    err = hipGetDevice(&prev);
    if (err == hipSuccess && prev == dev) prev = -1;
    else if (err == hipSuccess) err = hipSetDevice(dev);
  }
  ~DeviceGuard() {
    if (prev >= 0) (void)hipSetDevice(prev);
  }
};

}  // namespace fs
