// Host-side pieces of the C ABI: what every entry point asks of its arguments.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/ratsparse.h"
#include "common.h"

namespace rs {

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
inline size_t esize(int dtype) { return dtype == RS_BF16 ? 2 : 4; }
inline bool page_size_ok(int P) { return P == 16 || P == 32 || P == 64 || P == 128 || P == 256 || P == 512; }

// what a shape says of rows and heads; what B stands for is the caller's to look at
inline int check_rows(const rs_shape *s, bool need_page)
{
    if (!s) return RS_INVALID_ARG;
    if (s->B <= 0 || s->Hq <= 0 || s->Hkv <= 0 || s->Tcap <= 0) return RS_INVALID_ARG;
    if (s->Hq % s->Hkv != 0) return RS_INVALID_ARG;
    if (s->dtype != RS_F32 && s->dtype != RS_BF16) return RS_UNSUPPORTED;
    if (s->D != 64 && s->D != 128) return RS_UNSUPPORTED;
    if (need_page) {
        if (!page_size_ok(s->P)) return RS_UNSUPPORTED;
        if (s->Tcap % s->P != 0) return RS_INVALID_ARG;
    }
    if (s->Hq > kMaxUnits) return RS_UNSUPPORTED;
    return RS_OK;
}
// of calls in whose workspaces every head of every batch entry has control words
inline int check_shape(const rs_shape *s, bool need_page)
{
    const int st = check_rows(s, need_page);
    return st == RS_OK && (long)s->B * s->Hq > kMaxUnits ? RS_UNSUPPORTED : st;
}

inline int launch_status() { return hipGetLastError() == hipSuccess ? RS_OK : RS_LAUNCH_FAILED; }

}  // namespace rs
