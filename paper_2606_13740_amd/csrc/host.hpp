// What the library's translation units share on the host: errors and small arithmetic (arith.hpp).
#pragma once

#include <hip/hip_runtime.h>

#include <string>

#include "../../include/dllm.h"
#include "arith.hpp"

namespace dllm {

// Records msg as the thread's dllm_last_error() and returns code (dllm.hip).
int fail(int code, const std::string& msg);

// Every check of a dllm_select call, without a launch (batch.hip).
int select_check(const dllm_select_args* args);

// dllm_attention_paged; out_f32: d_out holds floats whatever the type (batch.hip).
int attention_paged(const dllm_attn_args* args, bool out_f32, hipStream_t s);

// An error that a call reports is taken from the runtime, so that the next call (or another library) does not
// find it and report it again.
#define HIP_TRY(expr)                                                                           \
    do {                                                                                        \
        hipError_t _e = (expr);                                                                 \
        if (_e != hipSuccess) {                                                                 \
            (void)hipGetLastError();                                                            \
            return fail(DLLM_E_HIP, std::string(#expr) + ": " + hipGetErrorString(_e));        \
        }                                                                                       \
    } while (0)

}  // namespace dllm
