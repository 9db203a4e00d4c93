/*
 * wsr_serve_internal.h - what the host side of libwsr_serve passes to its kernels: the public structures as they are
 * (checked), plus the launch plan where one is derived from them.
 */
#ifndef WSR_SERVE_INTERNAL_H
#define WSR_SERVE_INTERNAL_H

#include <hip/hip_runtime_api.h>

#include "wsr_serve.h"

namespace wsr_serve {

hipError_t launch_append(const wsr_qkv& p, hipStream_t s);

bool paged_fits(const wsr_paged& p);           /* one launch holds the call's units */
size_t paged_workspace(const wsr_paged& p);
hipError_t launch_paged(const wsr_paged& p, void* ws, hipStream_t s);

size_t logprobs_workspace(const wsr_logprobs& p);
hipError_t launch_logprobs(const wsr_logprobs& p, void* ws, hipStream_t s);

}  // namespace wsr_serve

#endif
