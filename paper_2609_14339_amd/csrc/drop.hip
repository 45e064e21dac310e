// Dropout of token rows, with the residual added in the same pass.
#include "drop.h"

namespace acsc {
namespace {

// A wave takes 512 columns of one row, eight a lane.  y = D(x) + residual: one
// rounding.  The gradient is the same call on dy.  HBM bounds it: 16384 x 8192
// bf16 with a residual 140 us, its 805 MB at 5.8 TB/s (partly from the caches);
// the draws, four 32-bit products a pair of values, stay beneath that.
template <typename T>
__global__ __launch_bounds__(256) void drop_kernel(const T *x, int64_t ldx, int64_t rows, int H, Drop d, const T *res,
                                                   int64_t ldr, T *y, int64_t ldy)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int segs = (H + 511) / 512;
    for (int64_t w = static_cast<int64_t>(blockIdx.x) * 4 + wave; w < rows * segs; w += static_cast<int64_t>(gridDim.x) * 4) {
        const int64_t row = w / segs;
        const int col = static_cast<int>(w - row * segs) * 512 + lane * 8, left = H - col;
        if (left <= 0)
            continue;
        float v[8], r[8];
        load8(x + row * ldx + col, left, v);
        if (res)
            load8(res + row * ldr + col, left, r);
        if (d.below)
            drop8(d, drop_row(d, row), col, v);
        if (res)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                v[i] += r[i];
        store8(y + row * ldy + col, left, v);
    }
}

inline int check_tensor(const void *p, int64_t rows, int64_t ld, int H, acsc_dtype dt, const char *name)
{
    ACSC_CHECK_ARG(rows == 0 || p, ACSC_EINVAL, "null pointer %s", name);
    ACSC_CHECK_ARG(ld >= H, ACSC_EINVAL, "ld of %s is %lld < %d columns", name, (long long)ld, H);
    ACSC_CHECK_ARG(aligned(p, dtype_size(dt)), ACSC_EALIGN, "%s not aligned to its elements", name);
    return ACSC_OK;
}

}  // namespace
}  // namespace acsc

using namespace acsc;

extern "C" int drop_apply(const void *x, acsc_dtype dt, int64_t rows, int H, int64_t ld_x, const drop_mask *drop,
                          const void *residual, int64_t ld_res, void *y, int64_t ld_y, hipStream_t stream)
{
    clear_error();
    ACSC_CHECK_ARG(dt == ACSC_F32 || dt == ACSC_BF16, ACSC_EDTYPE, "unknown dtype %d", (int)dt);
    ACSC_CHECK_ARG(rows >= 0 && rows < (1ll << 31), ACSC_EINVAL, "rows=%lld outside [0, 2^31)", (long long)rows);
    ACSC_CHECK_ARG(H >= 1 && H <= (1 << 22), ACSC_EINVAL, "H=%d outside [1, 2^22]", H);
    ACSC_CHECK_ARG(drop, ACSC_EINVAL, "null pointer drop");
    Drop d;
    if (int rc = drop_of(drop, rows, H, &d))
        return rc;
    if (int rc = check_tensor(x, rows, ld_x, H, dt, "x"))
        return rc;
    if (residual)
        if (int rc = check_tensor(residual, rows, ld_res, H, dt, "residual"))
            return rc;
    if (int rc = check_tensor(y, rows, ld_y, H, dt, "y"))
        return rc;
    ACSC_CHECK_ARG(y != x || rows == 0 || ld_y == ld_x, ACSC_EINVAL, "y in place of x needs ld_y == ld_x");
    ACSC_CHECK_ARG(y != residual || rows == 0 || ld_y == ld_res, ACSC_EINVAL, "y in place of the residual needs ld_y == ld_res");
    if (rows == 0)
        return ACSC_OK;
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>((rows * ((H + 511) / 512) + 3) / 4, 1 << 20)));
    if (dt == ACSC_BF16)
        ACSC_LAUNCH("drop_apply", drop_kernel<uint16_t>, grid, dim3(256), 0, stream, static_cast<const uint16_t *>(x), ld_x, rows,
                    H, d, static_cast<const uint16_t *>(residual), ld_res, static_cast<uint16_t *>(y), ld_y);
    else
        ACSC_LAUNCH("drop_apply", drop_kernel<float>, grid, dim3(256), 0, stream, static_cast<const float *>(x), ld_x, rows, H, d,
                    static_cast<const float *>(residual), ld_res, static_cast<float *>(y), ld_y);
    return check_launch("drop_apply");
}
