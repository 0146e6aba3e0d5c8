// What the translation units of the library share on the host: the device check, the library-owned memory and the
// thread's record of what a call took (all defined in flashdp_api.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/flashdp.h"

namespace flashdp {
namespace api {

__attribute__((visibility("hidden"))) int current_device(int* dev);
// At least `need` bytes of the library-owned workspace of the current device, grown if need be; FLASHDP_WORKSPACE_TOO_SMALL while `stream` is
// being captured.
__attribute__((visibility("hidden"))) int library_workspace(size_t need, hipStream_t stream, void** ptr);
// The same of memory apart from that workspace, for the activation that a call from 8-bit checkpoints unpacks.
__attribute__((visibility("hidden"))) int library_activation(size_t need, hipStream_t stream, void** ptr);
__attribute__((visibility("hidden"))) int schedule_of_call(int schedule);       // with FLASHDP_SCHEDULE in place of the argument, if set
__attribute__((visibility("hidden"))) int check_schedule_sizes(const flashdp_layer_t* layers, int n_layers, int64_t B, int64_t T, int dtype, int schedule);
__attribute__((visibility("hidden"))) int64_t compute_units();
__attribute__((visibility("hidden"))) int forward_override();   // FLASHDP_FORWARD, or -1
__attribute__((visibility("hidden"))) void note_kernel(const char* name);
__attribute__((visibility("hidden"))) hipError_t allow_lds(const void* kernel, int bytes);

}  // namespace api
}  // namespace flashdp
