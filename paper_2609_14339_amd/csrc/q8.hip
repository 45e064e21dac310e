// 8-bit activation checkpoints: coding a tensor and reading one back.
#include "q8.h"

namespace acsc {
namespace {

constexpr int kQThreads = 256;

inline int check_tensor(const void *p, int64_t rows, int64_t ld, int H, acsc_dtype dt, const char *name)
{
    ACSC_CHECK_ARG(rows == 0 || p, ACSC_EINVAL, "null pointer %s", name);
    ACSC_CHECK_ARG(ld >= H, ACSC_EINVAL, "ld of %s is %lld < %d columns", name, (long long)ld, H);
    ACSC_CHECK_ARG(aligned(p, dtype_size(dt)), ACSC_EALIGN, "%s not aligned to its elements", name);
    return ACSC_OK;
}

inline int check_shape(int64_t rows, int H, int dt)
{
    ACSC_CHECK_ARG(dt == ACSC_F32 || dt == ACSC_BF16, ACSC_EDTYPE, "unknown dtype %d", dt);
    ACSC_CHECK_ARG(rows >= 0 && rows < (1ll << 31), ACSC_EINVAL, "rows=%lld outside [0, 2^31)", (long long)rows);
    ACSC_CHECK_ARG(H >= 1 && H <= (1 << 22), ACSC_EINVAL, "H=%d outside [1, 2^22]", H);
    return ACSC_OK;
}

// A wave takes 512 columns of one row: eight per lane, so that a group is one
// row of 16 lanes.  HBM bounds it: 3 (bf16) bytes per value.
template <typename T>
__global__ __launch_bounds__(kQThreads) void q8_encode_kernel(const T *x, int64_t ldx, int64_t rows, int H, Q8 q)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int segs = (H + 511) / 512;
    for (int64_t w = static_cast<int64_t>(blockIdx.x) * 4 + wave; w < rows * segs; w += static_cast<int64_t>(gridDim.x) * 4) {
        const int64_t row = w / segs;
        const int col = static_cast<int>(w - row * segs) * 512 + lane * 8;
        float v[8];
        load8(x + row * ldx + col, H - col, v);
        uint32_t a = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            a = max(a, mag(v[i]));
        a = max16(a);
        float scale, inv;
        group_scale(a, scale, inv);
        if (col < H) {
            store_codes(q.codes + row * q.ldc + col, H - col, inv, v);
            if ((lane & 15) == 0)
                q.scales[row * q.lds + col / kGroup] = scale;
        }
    }
}

template <typename T>
__global__ __launch_bounds__(kQThreads) void q8_decode_kernel(Q8 q, int64_t rows, int H, int act, T *y, int64_t ldy)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int segs = (H + 511) / 512;
    for (int64_t w = static_cast<int64_t>(blockIdx.x) * 4 + wave; w < rows * segs; w += static_cast<int64_t>(gridDim.x) * 4) {
        const int64_t row = w / segs;
        const int col = static_cast<int>(w - row * segs) * 512 + lane * 8;
        if (col >= H)
            continue;
        float v[8];
        load_codes(q.codes + row * q.ldc + col, H - col, q.scales[row * q.lds + col / kGroup], v);
        apply_act<T>(v, act);
        store8(y + row * ldy + col, H - col, v);
    }
}

inline dim3 grid_of(int64_t rows, int H)
{
    const int64_t waves = rows * ((H + 511) / 512);
    return dim3(static_cast<unsigned>(std::min<int64_t>((waves + 3) / 4, 1 << 20)));
}

}  // namespace
}  // namespace acsc

using namespace acsc;

extern "C" int q8_encode(const void *x, acsc_dtype dt, int64_t rows, int H, int64_t ld_x, const q8_tensor *q,
                         hipStream_t stream)
{
    clear_error();
    if (int rc = check_shape(rows, H, dt))
        return rc;
    ACSC_CHECK_ARG(q, ACSC_EINVAL, "null checkpoint");
    if (int rc = check_tensor(x, rows, ld_x, H, dt, "x"))
        return rc;
    if (int rc = check_q8(q, rows, H))
        return rc;
    if (rows == 0)
        return ACSC_OK;
    if (dt == ACSC_BF16)
        ACSC_LAUNCH("q8_encode", q8_encode_kernel<uint16_t>, grid_of(rows, H), dim3(kQThreads), 0, stream,
                    static_cast<const uint16_t *>(x), ld_x, rows, H, q8_of(q));
    else
        ACSC_LAUNCH("q8_encode", q8_encode_kernel<float>, grid_of(rows, H), dim3(kQThreads), 0, stream,
                    static_cast<const float *>(x), ld_x, rows, H, q8_of(q));
    return check_launch("q8_encode");
}

extern "C" int q8_decode(const q8_tensor *q, int64_t rows, int H, acsc_act act, void *y, acsc_dtype dt, int64_t ld_y,
                         hipStream_t stream)
{
    clear_error();
    if (int rc = check_shape(rows, H, dt))
        return rc;
    if (int rc = check_act(act))
        return rc;
    ACSC_CHECK_ARG(q, ACSC_EINVAL, "null checkpoint");
    if (int rc = check_q8(q, rows, H))
        return rc;
    if (int rc = check_tensor(y, rows, ld_y, H, dt, "y"))
        return rc;
    if (rows == 0)
        return ACSC_OK;
    if (dt == ACSC_BF16)
        ACSC_LAUNCH("q8_decode", q8_decode_kernel<uint16_t>, grid_of(rows, H), dim3(kQThreads), 0, stream, q8_of(q), rows, H,
                    act, static_cast<uint16_t *>(y), ld_y);
    else
        ACSC_LAUNCH("q8_decode", q8_decode_kernel<float>, grid_of(rows, H), dim3(kQThreads), 0, stream, q8_of(q), rows, H, act,
                    static_cast<float *>(y), ld_y);
    return check_launch("q8_decode");
}
