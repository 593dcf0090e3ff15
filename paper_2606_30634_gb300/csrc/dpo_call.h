// dpo_call.h -- what the entry points that have no context share: their errors, where
// their buffers lie, and dpo_unpack8 as a step of dpo_ffn_backward.
#pragma once

#include "dpo.h"

#include <stdint.h>

namespace dpo {

// Sets the calling thread's message (dpo_last_error(NULL)) and returns code.
int call_fail(int code, const char *fmt, ...) __attribute__((format(printf, 2, 3)));

// Where a matrix lies: [lo, hi), in rows of `row` bytes, `pitch` bytes apart. Nothing for a
// null pointer or an empty matrix.
struct Extent {
    uintptr_t lo = 0, hi = 0, pitch = 0, row = 0;
};
inline Extent extent_of(const void *p, int64_t rows, int64_t cols, int64_t ld, int64_t size)
{
    if (p == nullptr || rows <= 0 || cols <= 0)
        return {};
    const uintptr_t b = reinterpret_cast<uintptr_t>(p);
    return {b, b + (uintptr_t)(((rows - 1) * ld + cols) * size), (uintptr_t)(ld * size),
            (uintptr_t)(cols * size)};
}
// Whether two share a byte. Blocks of columns of one buffer (equal pitches) may lie side by
// side; of matrices with different pitches what lies between the rows counts too.
inline bool overlap(const Extent &a, const Extent &b)
{
    if (a.lo >= b.hi || b.lo >= a.hi)
        return false;
    if (a.pitch != b.pitch)
        return true;
    const uintptr_t ab = a.lo <= b.lo ? (b.lo - a.lo) % a.pitch : a.pitch - (a.lo - b.lo - 1) % a.pitch - 1;
    return ab < a.row || ab + b.row > a.pitch;   // b's rows begin ab bytes into a's pitch
}

// dpo_unpack8 to bf16 beside the launch before it on the stream, which let its successor
// start early (launch_dependents) after its own wait, writes neither in nor out and does not
// read out: the kernel works first and waits for that launch at its end, so that what
// follows it, which it lets start early too, has both behind its own wait.
int unpack8_beside(const dpo_packed8 &in, int64_t rows, int64_t cols, void *out, void *cuda_stream);

}  // namespace dpo
