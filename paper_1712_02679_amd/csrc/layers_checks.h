// layers_checks.h -- argument checks that the calls of adacomp_layers.h and adacomp_sequence.h share (host code).
#pragma once

#include <cmath>
#include <cstddef>

#include "layers_plan.h"

namespace adacomp {

inline size_t element_bytes(uint32_t dtype) { return dtype == ADACOMP_DTYPE_F32 ? 4u : 2u; }
inline bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
inline size_t pad256(size_t x) { return (x + 255u) & ~size_t(255); }

inline int drop_args(const adacomp_dropout_t *drop, DropArgs &out)
{
    out = DropArgs();
    if (!drop) return ADACOMP_OK;
    if (!(drop->p >= 0.f && drop->p < 1.f) || drop->reserved != 0) return ADACOMP_EINVAL;
    const double threshold = std::floor(double(drop->p) * 65536.0 + 0.5);
    if (threshold >= 65536.0) return ADACOMP_EINVAL;
    if (!aligned(drop->step, 8)) return ADACOMP_EALIGN;
    out.step = drop->step;
    out.seed_lo = uint32_t(drop->seed);
    out.seed_hi = uint32_t(drop->seed >> 32);
    out.stream_lo = uint32_t(drop->stream);
    out.stream_hi = uint32_t(drop->stream >> 32);
    out.threshold = uint32_t(threshold);
    out.on = out.threshold != 0;
    out.factor = float(65536.0 / (65536.0 - threshold));
    return ADACOMP_OK;
}

inline int workspace_check(const void *workspace, size_t bytes, size_t needed)
{
    if (needed == 0) return ADACOMP_OK;
    if (!workspace) return ADACOMP_EINVAL;
    if (!aligned(workspace, 16)) return ADACOMP_EALIGN;
    return bytes < needed ? ADACOMP_EWORKSPACE : ADACOMP_OK;
}

}  // namespace adacomp
