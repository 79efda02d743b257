// Internal helpers shared by the library's translation units (not installed).
#pragma once
#include <cstdarg>
#include <cstdio>
#include <string>

#include "dpool.h"

namespace dpool {

// Record an error message for dp_last_error() and return `code`.
int fail(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
void clear_error();

// Validate a decode shape and report the workspace bytes its launch needs
// (paged_decode.hip): DP_OK, or the error code paged_decode_attention would
// return for the shape, with its message recorded.
int decode_workspace_bytes(const dp_decode_shape* shape, size_t* bytes);

// Enqueue window_prefill_attention of few rows over short windows as decode's
// one workgroup per segment does (paged_decode.hip); the arguments are valid.
// False, nothing enqueued, if the call is not such a one.
bool window_rows(const void* q, const void* k_blocks, const void* v_blocks, const int32_t* block_tables,
                 const int32_t* context_lens, const int32_t* q_start, float scale, int32_t window, int32_t n_sink,
                 const void* k_scale, const void* v_scale, void* out, const dp_prefill_shape* shape, void* stream);

}  // namespace dpool
