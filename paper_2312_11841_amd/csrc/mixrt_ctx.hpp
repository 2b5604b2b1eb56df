// The context and the error and launch handling that every entry point of the
// C ABI shares (defined in mixrt_api.cpp).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <string>

#include "mixrt.h"

struct mixrt_ctx {
    int device = 0;
    hipStream_t stream = nullptr;
    uint32_t flags = 0;
    int32_t tile_stripe = 0;
    int32_t early_stop_chunk = 0;
    int32_t block_levels = 0;
    unsigned int *work = nullptr;   // device: the render kernels' work counters
    int cus = 0;
    int64_t l2_bytes = 0;
    std::string err;
};

namespace mixrt {

extern thread_local std::string t_err;

// Records the message for the context (if any) and the thread, returns code.
int fail(mixrt_ctx *ctx, int code, const char *fmt, ...);
void clear_err(mixrt_ctx *ctx);
// Status of a launch; waits for it with MIXRT_FLAG_SYNC_CHECK.
int finish_launch(mixrt_ctx *ctx, hipError_t e, const char *what);
int bind_device(mixrt_ctx *ctx);

}  // namespace mixrt
