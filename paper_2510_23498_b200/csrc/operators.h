// Internal interface of the operators that work without a context: the gated linear recurrence (recurrence.cu), the residual step with its
// norms (residual.cu) and dropout (dropout.cu).  Their C entry points check the arguments and launch; nothing else of the library calls them.
#pragma once
#include "common.cuh"

namespace mpode {

// records the message that mpode_operator_error returns (per host thread) and passes the status through
mpode_status operator_fail(mpode_status s, const char* format, ...);
// after a launch: the runtime's refusal as a status
mpode_status operator_launched(cudaError_t e, const char* entry);

inline bool misaligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) != 0; }
inline bool known_dtype(mpode_dtype t) { return t == MPODE_F32 || t == MPODE_BF16 || t == MPODE_F16; }

// calls f with a value of the format's element type
template <typename F> inline cudaError_t with_low(mpode_dtype dt, F&& f) {
    if (dt == MPODE_F32) return f(float{});
    if (dt == MPODE_BF16) return f(__nv_bfloat16{});
    return f(__half{});
}

}  // namespace mpode
