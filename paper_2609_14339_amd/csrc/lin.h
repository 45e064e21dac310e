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
    int whole;        // tiles that are not cut along K; the rest is cut into
    int splits;       // pieces of kchunk each
    int kchunk;
    bool words_a, words_b;   // operands whose k (row) or indices (col) end inside a 16-byte chunk, not copied
    float *part;      // the pieces: of tiles [splits][tiles - whole][T][T]; of few tokens [splits][M][ldp], nullptr:
    int64_t ldp;      // one piece, through the epilogue
    const float *dbpart;   // weight gradient: slices of column sums of dz, [slices][M], that the product's first
    int slices;            // tiles add into db; nullptr: none
    float *db;
    Epi e;
};

// A kept input of the weight gradient: its checkpoint (or none: the tensor),
// and the activation that it still has to go through.
struct Kept {
    Q8 q;
    int act;
};

// Fragments of 16 rows of a wave, and waves, for a tile of TM rows and T columns.
constexpr int fragments(int TM) { return TM < 64 ? 1 : TM / 64; }
constexpr int waves(int TM, int T) { return TM / (16 * fragments(TM)) * (T < 128 ? 1 : T / 128); }

// What the epilogue reads beside the sums for eight columns of a row: the
// residual (forward), the kept pre-activation or its codes and scale (gate),
// or the output to add to (weight).
template <typename T>
struct Beside {
    Raw8<T> v;
    Codes8 codes;
    float scale;
};
template <typename T, int KIND>
__device__ __forceinline__ bool has_beside(const Epi &e)
{
    return KIND == kForward ? e.res != nullptr : KIND == kGate ? e.act != ACSC_ACT_NONE : e.accumulate != 0;
}
template <typename T, int KIND>
__device__ __forceinline__ void load_beside(const Epi &e, Beside<T> &b, int64_t m, int n, int left)
{
    const T *p = static_cast<const T *>(KIND == kForward ? e.res : KIND == kGate ? e.z : e.y);
    p += m * (KIND == kForward ? e.ldr : KIND == kGate ? e.ldz : e.ldy) + n;
    if (KIND != kGate) {
        load_raw(p, left, b.v);
        return;
    }
    // written once, after both ways: in each of them, b stays in memory
    Beside<T> r = {};
    if (e.q.codes) {
        load_raw(e.q.codes + m * e.q.ldc + n, left, r.codes);
        r.scale = left > 0 ? e.q.scales[m * e.q.lds + n / kGroup] : 0.f;
    } else {
        load_raw(p, left, r.v);
    }
    b = r;
}
template <typename T, int KIND>
__device__ __forceinline__ void beside_values(const Epi &e, const Beside<T> &b, float (&v)[8])
{
    if (KIND == kGate && e.q.codes) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = code_value(b.codes.at(i), b.scale);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = b.v.at(i);
    }
}

// Eight values of row m at columns n .. n + 7 (n a multiple of 8; the first
// `left` of them exist, none of a row past the end) through the epilogue.
// Sixteen lanes of the wave, aligned, hold one group of 128 columns of a row,
// and every lane of the wave calls it.  T is the type of y, z, bias and
// residual; `bias` holds the eight columns', zeros without one.
template <typename T, int KIND>
__device__ __forceinline__ void epilogue(const Epi &e, float (&v)[8], const float (&bias)[8], const Beside<T> &beside,
                                         int64_t m, int n, int left)
{
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
                a = max(a, i < left ? mag(v[i]) : 0u);
            a = max16(a);
            float scale, inv;
            group_scale(a, scale, inv);
            store_codes(e.q.codes + m * e.q.ldc + n, left, inv, v);
            if (left > 0 && n % kGroup == 0)
                e.q.scales[m * e.q.lds + n / kGroup] = scale;
        }
        apply_act<T>(v, e.act);
    }
    if (has_beside<T, KIND>(e)) {
        float b[8];
        beside_values<T, KIND>(e, beside, b);
        if (KIND == kGate) {
            apply_slope<T>(v, b, e.act);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                v[i] += b[i];
        }
    }
    store8(static_cast<T *>(e.y) + m * e.ldy + n, left, v);
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
// 256 (bf16) contiguous bytes, four a step.  What the epilogue reads leaves
// for four steps at once (one at a time each waits a memory latency: a
// residual on 16384 x 2048 -> 8192 cost 100 us that way, see the forward
// kernel's figures); WHOLE: the wave's 128 columns all exist.
template <typename T, int KIND, int NA, bool WHOLE>
__device__ __forceinline__ void put_rows(const Gemm &g, const char *lds, int64_t m0, int n0, int end)
{
    const int lane = threadIdx.x & 63, n = n0 + (lane & 15) * 8;
    const int cols = WHOLE ? 8 : end - n;
    float bias[8];
    load_bias<T, KIND>(g.e, n, g.N, bias);
#pragma unroll 1
    for (int r0 = 0; r0 < NA * 4; r0 += 4) {
        Beside<T> beside[4];
        if (has_beside<T, KIND>(g.e)) {
#pragma unroll
            for (int u = 0; u < 4; ++u)
                load_beside<T, KIND>(g.e, beside[u], min<int64_t>(m0 + (r0 + u) * 4 + (lane >> 4), g.M - 1), n, cols);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int row = (r0 + u) * 4 + (lane >> 4), c = (lane & 15) * 2;
            const f32x4 lo = *reinterpret_cast<const f32x4 *>(lds + row * 512 + (c ^ (row & 31)) * 16);
            const f32x4 hi = *reinterpret_cast<const f32x4 *>(lds + row * 512 + ((c + 1) ^ (row & 31)) * 16);
            float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
            const int64_t m = m0 + row;
            const int left = m < g.M ? cols : 0;
            epilogue<T, KIND>(g.e, v, bias, beside[u], m, n, left);
        }
    }
}
// The first column of tiles adds the slices of db, in order.
template <int KIND>
__device__ __forceinline__ void put_db(const Gemm &g, int64_t m0, int rows)
{
    if (KIND != kWeight || !g.dbpart)
        return;
    for (int64_t m = m0 + threadIdx.x; m < min<int64_t>(g.M, m0 + rows); m += blockDim.x) {
        float s = 0.f;
#pragma unroll 8
        for (int i = 0; i < g.slices; ++i)
            s += g.dbpart[i * g.M + m];
        g.db[m] = g.e.accumulate ? g.db[m] + s : s;
    }
}

// The tile's columns stop at `end`.  `part`: the piece's rows and columns of
// this wave, ld a row, or nullptr.
template <typename T, int KIND, int NA>
__device__ __forceinline__ void put_tile(const Gemm &g, const f32x4 (&acc)[NA][8], char *lds, int64_t m0, int n0,
                                         int end, float *part, int ld)
{
    const int lane = threadIdx.x & 63;
    if (part) {
        // four consecutive columns a lane, 64 bytes of a row at a time
#pragma unroll
        for (int a = 0; a < NA; ++a)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j * 16 < ld)
                    *reinterpret_cast<f32x4 *>(part + (a * 16 + (lane & 15)) * ld + j * 16 + (lane >> 4) * 4) = acc[a][j];
        return;
    }
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
    if (n0 + 128 <= end)
        put_rows<T, KIND, NA, true>(g, lds, m0, n0, end);
    else
        put_rows<T, KIND, NA, false>(g, lds, m0, n0, end);
}

// Tile `id` of the product's order: bands of four rows of tiles, column by
// column, so that what an XCD's CUs read together stays in its L2.
__device__ __forceinline__ void tile_at(const Gemm &g, int64_t id, int &tile_m, int &tile_n)
{
    const int64_t band = id / (4 * g.tn), in = id - band * 4 * g.tn;
    const int height = static_cast<int>(min<int64_t>(g.tm - band * 4, 4));
    tile_m = static_cast<int>(band * 4 + in % height);
    tile_n = static_cast<int>(in / height);
}

}  // namespace acsc
