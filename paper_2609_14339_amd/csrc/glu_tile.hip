// The tiled products of the gated linear layer, by the linear layers' kernel:
// forward with rows of the gate's and of the up projection's weights in every
// tile, 64 of each in turn, so that a lane ends with both pre-activations of
// its columns; and the gradient through the gate and the product.
#include "lin_plan.h"
#include "lin_tile.h"

namespace acsc {
namespace {

template <typename E, int TM, int T>
int launch_kind(const Gemm &g, EpiKind kind, hipStream_t st, const char *tag)
{
    if constexpr (T >= 128)
        if (kind == kGluForward)
            return launch<E, TM, T, false, false, kGluForward, E>(g, st, tag);
    return launch<E, TM, T, false, true, kGluGate, E>(g, st, tag);
}

template <typename E>
int launch_tile(const Gemm &g, int rows, int cols, EpiKind kind, hipStream_t st, const char *tag)
{
    if (cols == 64)
        return launch_kind<E, 128, 64>(g, kind, st, tag);
    if (rows == 128)
        return launch_kind<E, 128, 128>(g, kind, st, tag);
    return rows == 64 ? launch_kind<E, 64, 128>(g, kind, st, tag) : launch_kind<E, 32, 128>(g, kind, st, tag);
}

}  // namespace

int glu_tile_run(const Gemm &g, int rows, int cols, EpiKind kind, acsc_dtype dt, hipStream_t st, const char *tag)
{
    if (dt == ACSC_F32)
        return launch_tile<float>(g, rows, cols, kind, st, tag);
    return rows == 256 ? launch_kind<uint16_t, 256, 256>(g, kind, st, tag) : launch_tile<uint16_t>(g, rows, cols, kind, st, tag);
}

}  // namespace acsc
