// The tiled products of the gated linear layer, by the linear layers' kernel:
// forward with rows of the gate's and of the up projection's weights in every
// tile, 64 of each in turn, so that a lane ends with both pre-activations of
// its columns; and the gradient through the gate and the product.
//
// What bounds them: the products as in the plain layers (8192 x 8192 -> 28672
// bf16 5300 to 5400 us, 1430 TFLOP/s, z kept), and epilogues that one workgroup
// a CU cannot hide: 16384 x 2048 -> 8192 takes 840 us, 920 with z kept (537 MB)
// and 950 with codes (268 MB and their arithmetic); the gradient of 8192 x 4096
// -> 14336 730 as a plain product and 850 with two checkpoints read and dz and h
// written, 700 MB more, which HBM moves in 137.
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
