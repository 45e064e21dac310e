// Dropout as kernels take it: every value's draw comes from the step's key
// again, so no mask is stored.
#pragma once

#include "prf.h"
#include "q8.h"

namespace acsc {

struct Drop {
    uint64_t key;
    uint32_t below;   // a value is kept where its 16 bits are below; 0: no dropout
    float up;         // the factor of kept values, 65536 / below
};

// Host checks, and the mask's key.  The chain over the key's fields goes on
// with "drop" and the site, so no dropout shares draws with a boundary's mask
// of the same fields or with another site.
inline int drop_of(const drop_mask *m, int64_t rows, int H, Drop *d)
{
    *d = Drop{0, 0, 1.f};
    if (!m)
        return ACSC_OK;
    ACSC_CHECK_ARG(m->p >= 0.0 && m->p < 1.0, ACSC_EINVAL, "p=%g outside [0, 1)", m->p);
    ACSC_CHECK_ARG(m->key.H == static_cast<uint32_t>(H), ACSC_EINVAL, "key.H=%u != H=%d", m->key.H, H);
    ACSC_CHECK_ARG(static_cast<uint64_t>(m->key.B) * m->key.S == static_cast<uint64_t>(rows), ACSC_EINVAL,
                   "rows=%lld != key.B*key.S=%llu", (long long)rows, (unsigned long long)m->key.B * m->key.S);
    uint32_t T = 0;
    if (int rc = iid_threshold(1.0 - m->p, &T))
        return rc;
    if (T == 65536)
        return ACSC_OK;   // keeps every value
    *d = Drop{mix64((chain_key(m->key) ^ (0x64726F7000000000ull | m->site)) + kGamma), T, 65536.f / static_cast<float>(T)};
    return ACSC_OK;
}

struct DropRow {
    uint32_t a, b;
};
__device__ __forceinline__ DropRow drop_row(const Drop &d, int64_t row)
{
    const uint64_t k = mix64((d.key ^ static_cast<uint64_t>(row)) + kGamma);
    return {static_cast<uint32_t>(k), static_cast<uint32_t>(k >> 32)};
}

// Eight values at columns col .. col + 7 (col a multiple of 8): kept ones times
// the factor, +0 in the others' place whatever they hold.
__device__ __forceinline__ void drop8(const Drop &d, const DropRow &r, int col, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t h = iid_pair(r.a, r.b, static_cast<uint32_t>(col / 2 + i));
        v[2 * i] = (h & 0xFFFFu) < d.below ? v[2 * i] * d.up : 0.f;
        v[2 * i + 1] = (h >> 16) < d.below ? v[2 * i + 1] * d.up : 0.f;
    }
}

}  // namespace acsc
