// Argument checks shared by the C entry points; none makes a HIP call.
#pragma once

#include <string.h>

#include "dyad.h"

namespace dyad {
namespace abi {

constexpr int64_t kMaxDim = (int64_t)1 << 31;   // any single width or token count
constexpr int64_t kMaxElems = (int64_t)1 << 40; // any single tensor, in elements

// Per-block size; a width that D does not divide is zero-padded up to D blocks.
inline int64_t block(int64_t n, int64_t D) { return (n + D - 1) / D; }

// The int a caller passed for an enum parameter.  A C caller may pass any
// int there; reading the parameter through its enum type would be undefined
// in C++ for values outside the enumerators' range, so its bytes are read as
// an int and every check works on that.
template <class E>
int enum_value(const E &e) {
    static_assert(sizeof(E) == sizeof(int), "C enums are int-sized");
    int v;
    memcpy(&v, &e, sizeof v);
    return v;
}

inline bool aligned16(const void *p) { return p == nullptr || ((uintptr_t)p & 15u) == 0; }

inline int check_sizes(int variant, int64_t n_in, int64_t n_out, int64_t D, int64_t M, int dtype) {
    if (variant != DYAD_IT && variant != DYAD_OT && variant != DYAD_DT) return DYAD_ERR_INVALID_ARG;
    if (dtype != DYAD_F32 && dtype != DYAD_BF16) return DYAD_ERR_DTYPE;
    if (n_in <= 0 || n_out <= 0 || D <= 0 || M < 0) return DYAD_ERR_INVALID_ARG;
    if (n_in >= kMaxDim || n_out >= kMaxDim || M >= kMaxDim) return DYAD_ERR_INVALID_ARG;
    if (M * n_in >= kMaxElems || M * n_out >= kMaxElems) return DYAD_ERR_INVALID_ARG;
    if (D >= kMaxDim || D * block(n_in, D) * block(n_out, D) >= kMaxElems) return DYAD_ERR_INVALID_ARG;
    return DYAD_OK;
}

inline bool in_transposed(int v) { return v == DYAD_IT || v == DYAD_DT; }
inline bool out_transposed(int v) { return v == DYAD_OT || v == DYAD_DT; }

inline int launch_status(hipError_t e) { return e == hipSuccess ? DYAD_OK : DYAD_ERR_LAUNCH; }

}  // namespace abi
}  // namespace dyad
