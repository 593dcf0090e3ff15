// dpo_call.h -- what the entry points that have no context share: their errors, and
// dpo_unpack8 as a step of dpo_ffn_backward.
#pragma once

#include "dpo.h"

namespace dpo {

// Sets the calling thread's message (dpo_last_error(NULL)) and returns code.
int call_fail(int code, const char *fmt, ...) __attribute__((format(printf, 2, 3)));

// dpo_unpack8 to bf16 beside the launch before it on the stream, which let its successor
// start early (launch_dependents) after its own wait, writes neither in nor out and does not
// read out: the kernel works first and waits for that launch at its end, so that what
// follows it, which it lets start early too, has both behind its own wait.
int unpack8_beside(const dpo_packed8 &in, int64_t rows, int64_t cols, void *out, void *cuda_stream);

}  // namespace dpo
