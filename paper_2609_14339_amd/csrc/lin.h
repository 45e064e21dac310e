// What the kernels of the linear layers share: operands, the epilogue, and
// the plan that cuts a product into tiles and pieces.
#pragma once

#include "q8.h"

namespace acsc {

typedef float f32x4 __attribute__((ext_vector_type(4)));

// C [M, N] = sum over k of A(m, k) B(n, k).  An operand is stored with k
// contiguous ("row": p[m * ld + k]) or with its own index contiguous ("col":
// p[k * ld + m]); the three products of a layer are
//   forward  A = x row, B = W row;   input gradient  A = dz row, B = W col;
//   weight gradient  A = dz col, B = x col.
struct Operand {
    const void *p;
    int64_t ld;
};

// Epilogues.  Forward: z = C + bias, kept whole or coded, then act(z) +
// residual.  Gate: C act'(z) of a kept z.  Weight: C, or added to the output.
enum EpiKind { kForward = 0, kGate = 1, kWeight = 2 };

struct Epi {
    void *y;
    int64_t ldy;
    const void *bias;
    const void *res;
    int64_t ldr;
    void *z;          // forward: out or nullptr; gate: in or nullptr
    int64_t ldz;
    Q8 q;             // forward: out or none; gate: in or none
    int act;
    int accumulate;
};

struct Gemm {
    Operand A, B;
    int64_t M;
    int N, K;
    int tm, tn;       // tiles along M and N
    int splits;       // pieces along K, kchunk each
    int kchunk;
    float *part;      // piece s at part + s * M * ldp; nullptr: one piece, through the epilogue
    int64_t ldp;
    Epi e;
};

// Eight values of row m at columns n .. n + 7 (n a multiple of 8) through the
// epilogue.  Sixteen lanes of the wave, aligned, hold one group of 128
// columns of a row, and every lane of the wave calls it (`on`: the row
// exists); T is the type of y, z, bias and residual, `bias` the eight columns'
// (zeros without one).
template <typename T, int KIND>
__device__ __forceinline__ void epilogue(const Epi &e, float (&v)[8], const float (&bias)[8], bool on, int64_t m, int n,
                                         int N)
{
    const int left = on ? N - n : 0;
    if (KIND == kForward) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] += bias[i];
        if (e.z)
            store8(static_cast<T *>(e.z) + m * e.ldz + n, left, v);
        if (e.q.codes) {
            uint32_t a = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < left)
                    a = max(a, mag(v[i]));
            a = max16(a);
            float scale, inv;
            group_scale(a, scale, inv);
            store_codes(e.q.codes + m * e.q.ldc + n, left, inv, v);
            if (left > 0 && n % kGroup == 0)
                e.q.scales[m * e.q.lds + n / kGroup] = scale;
        }
        apply_act<T>(v, e.act);
        if (e.res) {
            float b[8];
            load8(static_cast<const T *>(e.res) + m * e.ldr + n, left, b);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                v[i] += b[i];
        }
    }
    if (left <= 0)
        return;
    if (KIND == kGate && e.act != ACSC_ACT_NONE) {
        float z[8];
        if (e.q.codes)
            load_codes(e.q.codes + m * e.q.ldc + n, left, e.q.scales[m * e.q.lds + n / kGroup], z);
        else
            load8(static_cast<const T *>(e.z) + m * e.ldz + n, left, z);
        apply_slope<T>(v, z, e.act);
    }
    T *y = static_cast<T *>(e.y) + m * e.ldy + n;
    if (KIND == kWeight && e.accumulate) {
        float o[8];
        load8(y, left, o);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] += o[i];
    }
    store8(y, left, v);
}

template <typename T, int KIND>
__device__ __forceinline__ void load_bias(const Epi &e, int n, int N, float (&b)[8])
{
    if (KIND == kForward)
        load8(static_cast<const T *>(e.bias) + n, e.bias ? N - n : 0, b);
}

// A wave's accumulators of 16 NA rows by 128 columns through the epilogue, or
// into a piece of a cut product.  acc[a][j] holds in lane L the columns
// 16 j + 4 (L / 16) + i of row 16 a + L % 16; they turn into runs of eight
// columns in `lds` (8 KiB NA, the wave's own), whose 16-byte chunks are
// XOR-swizzled by the row so that neither side conflicts: rows then go out as
// 256 (bf16) contiguous bytes.
template <typename T, int KIND, int NA>
__device__ __forceinline__ void put_rows(const Gemm &g, const f32x4 (&acc)[NA][8], char *lds, int64_t m0, int n0,
                                         int split)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int a = 0; a < NA; ++a)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int row = a * 16 + (lane & 15), chunk = (j * 4 + (lane >> 4)) ^ (row & 31);
            *reinterpret_cast<f32x4 *>(lds + row * 512 + chunk * 16) = acc[a][j];
        }
    // the wave reads what its own lanes wrote: LDS keeps a wave's order
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    const int n = n0 + (lane & 15) * 8;
    float bias[8];
    if (!g.part)
        load_bias<T, KIND>(g.e, n, g.N, bias);
#pragma unroll 1
    for (int r = 0; r < NA * 4; ++r) {
        const int row = r * 4 + (lane >> 4), c = (lane & 15) * 2;
        const f32x4 lo = *reinterpret_cast<const f32x4 *>(lds + row * 512 + (c ^ (row & 31)) * 16);
        const f32x4 hi = *reinterpret_cast<const f32x4 *>(lds + row * 512 + ((c + 1) ^ (row & 31)) * 16);
        float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        const int64_t m = m0 + row;
        if (g.part)
            store8(g.part + (split * g.M + m) * g.ldp + n, m < g.M ? g.N - n : 0, v);
        else
            epilogue<T, KIND>(g.e, v, bias, m < g.M, m, n, g.N);
    }
}

}  // namespace acsc
