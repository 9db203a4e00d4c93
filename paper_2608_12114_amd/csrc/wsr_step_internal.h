/*
 * wsr_step_internal.h - what the host side of libwsr_step passes to its kernels: the public structures
 * as they are (checked), plus the launch plan where one is derived from them.
 */
#ifndef WSR_STEP_INTERNAL_H
#define WSR_STEP_INTERNAL_H

#include <stdint.h>
#include <hip/hip_runtime_api.h>

#include "wsr_step.h"

namespace wsr_step {

/* Workgroups of a launch at most: one of 2^32 threads or more is cut to what is left over 2^32, without an error. */
constexpr int64_t most_blocks(int threads) { return UINT32_MAX / threads; }

hipError_t launch_block_norm(const wsr_block& p, hipStream_t s);

size_t lora_workspace(const wsr_lora* mods, int32_t n, int32_t n_tokens);
hipError_t launch_lora(const wsr_lora* mods, int32_t n, int32_t n_tokens, const int32_t* adapter_of, int32_t n_adapters,
                       const int32_t* ranks, const float* scales, void* ws, hipStream_t s);

bool attn_fits(const wsr_attn& p);            /* one launch holds the call's row tiles */
size_t attn_workspace(const wsr_attn& p);
hipError_t launch_attn(const wsr_attn& p, void* ws, hipStream_t s);

size_t verify_workspace(const wsr_verify& p);
hipError_t launch_verify(const wsr_verify& p, void* ws, hipStream_t s);

}  // namespace wsr_step

#endif
