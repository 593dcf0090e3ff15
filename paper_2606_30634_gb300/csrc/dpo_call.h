// dpo_call.h -- errors of the entry points that have no context.
#pragma once

namespace dpo {

// Sets the calling thread's message (dpo_last_error(NULL)) and returns code.
int call_fail(int code, const char *fmt, ...) __attribute__((format(printf, 2, 3)));

}  // namespace dpo
