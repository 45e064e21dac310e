// The tiled products of the linear layers (the kernel and its figures are in
// lin_tile.h).
#include "lin_plan.h"
#include "lin_tile.h"

namespace acsc {
namespace {

template <typename E, int TM, int T>
int launch_kind(const Gemm &g, EpiKind kind, acsc_dtype out, hipStream_t st, const char *tag)
{
    if (kind == kForward)
        return launch<E, TM, T, false, false, kForward, E>(g, st, tag);
    if (kind == kGate)
        return launch<E, TM, T, false, true, kGate, E>(g, st, tag);
    if constexpr (TM >= 64)
        return out == ACSC_BF16 ? launch<E, TM, T, true, true, kWeight, uint16_t>(g, st, tag)
                                : launch<E, TM, T, true, true, kWeight, float>(g, st, tag);
    return ACSC_EINVAL;   // tiles of 32 rows are of the other two kinds
}

template <typename E>
int launch_tile(const Gemm &g, int rows, int cols, EpiKind kind, acsc_dtype out, hipStream_t st, const char *tag)
{
    if (cols == 64)
        return launch_kind<E, 128, 64>(g, kind, out, st, tag);
    if (rows == 128)
        return launch_kind<E, 128, 128>(g, kind, out, st, tag);
    return rows == 64 ? launch_kind<E, 64, 128>(g, kind, out, st, tag) : launch_kind<E, 32, 128>(g, kind, out, st, tag);
}

}  // namespace

int lin_tile_run(const Gemm &g, int rows, int cols, EpiKind kind, acsc_dtype dt, acsc_dtype out, hipStream_t st,
                 const char *tag)
{
    if (dt == ACSC_F32)
        return launch_tile<float>(g, rows, cols, kind, out, st, tag);
    return rows == 256 ? launch_kind<uint16_t, 256, 256>(g, kind, out, st, tag)
                       : launch_tile<uint16_t>(g, rows, cols, kind, out, st, tag);
}

}  // namespace acsc
