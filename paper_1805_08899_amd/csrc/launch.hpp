// What every launch of the newer entry points goes through: a pending HIP error of earlier, unrelated calls is cleared, the launch is
// bracketed by events while profiling is on, and its error becomes the calling thread's last error.
//
//     LaunchRecord r = launch_begin("embed_fwd", st);
//     k_embed_fwd<<<...>>>(...);
//     if (echo_status_t s = launch_end(r)) return s;
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/echoattn.h"

namespace echo {

struct LaunchRecord {
    const char *name;
    hipStream_t st;
    hipEvent_t t0, t1;
};
LaunchRecord launch_begin(const char *name, hipStream_t st);
echo_status_t launch_end(LaunchRecord &r);

}  // namespace echo
