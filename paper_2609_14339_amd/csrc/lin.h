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
    float *part;      // splits > 1: piece s at part + s * M * ldp
    int64_t ldp;
    float *dbpart;    // weight gradient with db: piece s at dbpart + s * M, else nullptr
    Epi e;
};

// One row's values at columns n0 + 16 j .. n0 + 16 j + 3 (j < NJ), through the
// epilogue.  With NJ = 8 the four lanes 16 apart hold one group of 128
// columns of the row; with NJ = 1 a run of 32 lanes does.  Every lane of the
// wave calls it (`on`: its row exists); T is the type of y, z, bias and
// residual.
template <typename T, int KIND, int NJ>
__device__ __forceinline__ void epilogue(const Epi &e, float (&v)[NJ][4], bool on, int64_t m, int n0, int N)
{
    if (KIND == kForward) {
        if (e.bias) {
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                float b[4];
                load4(static_cast<const T *>(e.bias) + n0 + 16 * j, N - n0 - 16 * j, b);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    v[j][i] += b[i];
            }
        }
        if (e.z && on) {
            T *z = static_cast<T *>(e.z) + m * e.ldz;
#pragma unroll
            for (int j = 0; j < NJ; ++j)
                store4(z + n0 + 16 * j, N - n0 - 16 * j, v[j]);
        }
        if (e.q.codes) {
            uint32_t a = 0;
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (n0 + 16 * j + i < N)
                        a = max(a, mag(v[j][i]));
            if (NJ == 1)
                a = max16(a);
            a = max(a, static_cast<uint32_t>(__shfl_xor(static_cast<int>(a), 16)));
            if (NJ > 1)
                a = max(a, static_cast<uint32_t>(__shfl_xor(static_cast<int>(a), 32)));
            float scale, inv;
            group_scale(a, scale, inv);
            if (on) {
                int8_t *c = e.q.codes + m * e.q.ldc;
#pragma unroll
                for (int j = 0; j < NJ; ++j)
                    store_codes(c + n0 + 16 * j, N - n0 - 16 * j, inv, v[j]);
                if (n0 < N && n0 % kGroup == 0)
                    e.q.scales[m * e.q.lds + n0 / kGroup] = scale;
            }
        }
        if (e.act != ACSC_ACT_NONE) {
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    v[j][i] = act_value(v[j][i], e.act);
        }
        if (e.res && on) {
            const T *r = static_cast<const T *>(e.res) + m * e.ldr;
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                float b[4];
                load4(r + n0 + 16 * j, N - n0 - 16 * j, b);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    v[j][i] += b[i];
            }
        }
    }
    if (!on)
        return;
    if (KIND == kGate && e.act != ACSC_ACT_NONE) {
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            const int n = n0 + 16 * j;
            if (n < N) {
                float z[4];
                if (e.q.codes)
                    load_codes(e.q.codes + m * e.q.ldc + n, N - n, e.q.scales[m * e.q.lds + n / kGroup], z);
                else
                    load4(static_cast<const T *>(e.z) + m * e.ldz + n, N - n, z);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    v[j][i] *= act_slope(z[i], e.act);
            }
        }
    }
    T *y = static_cast<T *>(e.y) + m * e.ldy;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
        const int n = n0 + 16 * j;
        if (KIND == kWeight && e.accumulate) {
            float o[4];
            load4(y + n, N - n, o);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                v[j][i] += o[i];
        }
        store4(y + n, N - n, v[j]);
    }
}

}  // namespace acsc
