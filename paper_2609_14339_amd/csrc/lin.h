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
// The gated product's, with rows of B for the gate and, F after each, for the
// up projection: GluForward: g, u = C + bias, kept whole or coded, then
// act(g) u.  GluGate: (C u act'(g), C act(g)) of kept g and u, and act(g) u.
enum EpiKind { kForward = 0, kGate = 1, kWeight = 2, kGluForward = 3, kGluGate = 4 };

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
    // The gated product's: z [rows, 2 F] (gate, then up) or q and q_up, out
    // (forward, where y is the hidden activation) or in (gate, where y is
    // [rows, 2 F] and hidden an output or nullptr).
    Q8 q_up;
    void *hidden;
    int64_t ldh;
    // gate: column sums of both halves of y before their rounding, or nullptr: a
    // partial of each row of tiles, [tm][2][F], and behind them those of cut tiles,
    // `cut_slots` of each row of tiles from cut_first on
    float *sums;
    int cut_first, cut_slots;
};

struct Gemm {
    Operand A, B;
    int64_t M;
    int N, K;         // kGluForward: N = F, and B has 2 F rows
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

// a = act(g) and s = act'(g), eight at a time, from one exponential.
template <typename T>
__device__ __forceinline__ void act_both(const float (&g)[8], int act, float (&a)[8], float (&s)[8])
{
    const auto each = [&](auto one) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            one(g[i], a[i], s[i]);
    };
    if (act == ACSC_ACT_SILU)
        each([](float z, float &a, float &s) {
            float t, c;
            sigmoid<T>(z, t, c);
            a = z * t;
            s = t * __builtin_fmaf(z, c, 1.f);
        });
    else if (act == ACSC_ACT_GELU)
        each([](float z, float &a, float &s) {
            float e;
            const float q = normal_tail<T>(z, e);
            a = __builtin_fmaf(-fabsf(z > 64.f ? 64.f : z), q, z < 0.f ? 0.f : z);
            s = __builtin_fmaf(z * 0.39894228040143268f, e, z < 0.f ? q : 1.f - q);
        });
    else if (act == ACSC_ACT_RELU)
        each([](float z, float &a, float &s) {
            a = act_value<float>(z, ACSC_ACT_RELU);
            s = act_slope<float>(z, ACSC_ACT_RELU);
        });
    else
        each([](float z, float &a, float &s) {
            a = z;
            s = 1.f;
        });
}

// The largest magnitude of the first `left` of eight values.
__device__ __forceinline__ uint32_t mag8(const float (&v)[8], int left)
{
    uint32_t a = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        a = max(a, i < left ? mag(v[i]) : 0u);
    return a;
}
// What the other half of sixteen lanes holds (row_ror 8).
__device__ __forceinline__ float other8(float x)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x128, 0xF, 0xF, false));
}

// Where eight columns n .. n + 7 of row m of what the gated epilogues read and
// write lie; a step of rows adds uniform strides (the 64-bit products of every
// row's addresses took a quarter of the epilogue).
template <typename T>
struct GluAt {
    int8_t *cg, *cu;      // codes, or nullptr
    float *sg, *su;
    T *z, *y, *h;
    __device__ __forceinline__ GluAt(const Epi &e, int64_t m, int n)
    {
        cg = e.q.codes + m * e.q.ldc + n;
        cu = e.q_up.codes + m * e.q_up.ldc + n;
        sg = e.q.scales + m * e.q.lds + n / kGroup;
        su = e.q_up.scales + m * e.q_up.lds + n / kGroup;
        z = static_cast<T *>(e.z) + m * e.ldz + n;
        y = static_cast<T *>(e.y) + m * e.ldy + n;
        h = static_cast<T *>(e.hidden) + m * e.ldh + n;
    }
    __device__ __forceinline__ void step(const Epi &e, int rows)
    {
        cg += rows * e.q.ldc;
        cu += rows * e.q_up.ldc;
        sg += rows * e.q.lds;
        su += rows * e.q_up.lds;
        z += rows * e.ldz;
        y += rows * e.ldy;
        h += rows * e.ldh;
    }
};

// The gated product forward: eight columns from n on of a row of g and u
// through the epilogue; `left` of them exist (WHOLE: all, of a row that does).
// With a checkpoint sixteen lanes of the wave, aligned, hold a group of 128 columns of both; half of them forms
// the gate's scale, the other the up projection's.
template <typename T, bool CODES = true, bool WHOLE = false>
__device__ __forceinline__ void glu_epilogue(const Epi &e, int F, float (&g)[8], float (&u)[8], const GluAt<T> &at, int n, int left)
{
    if (e.z) {
        store8(at.z, left, g);
        store8(at.z + F, left, u);
    }
    if (CODES && e.q.codes) {
        const bool low = (threadIdx.x & 8) == 0;
        const uint32_t ag = max16(mag8(g, WHOLE ? 8 : left)), au = max16(mag8(u, WHOLE ? 8 : left));
        float scale, inv;
        group_scale(low ? ag : au, scale, inv);
        const float inv2 = other8(inv), scale2 = other8(scale);
        store_codes(at.cg, left, low ? inv : inv2, g);
        store_codes(at.cu, left, low ? inv2 : inv, u);
        if (left > 0 && n % kGroup == 0) {
            *at.sg = scale;
            *at.su = scale2;
        }
    }
    apply_act<T>(g, e.act);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        g[i] *= u[i];
    store8(at.y, left, g);
}
template <typename T>
__device__ __forceinline__ void glu_bias(const Epi &e, int F, int n, float (&bg)[8], float (&bu)[8])
{
    const T *b = static_cast<const T *>(e.bias) + n;
    load8(b, e.bias ? F - n : 0, bg);
    load8(b + F, e.bias ? F - n : 0, bu);
}

// The gated product's gradient: eight columns of row m of dh = C through the
// epilogue, from kept g and u.  sg, su: what is added to their column sums.
// Kept values as they are stored, of either form in the same registers (in two
// sets of their own 8192 x 4096 -> 14336 from codes took 878 us, 868 so).
template <typename T>
struct GluBeside {
    static constexpr int W = sizeof(T) * 2;
    uint32_t g[W], u[W];
    float sg, su;
};
template <typename T>
__device__ __forceinline__ void load_glu_beside(const Epi &e, int F, GluBeside<T> &b, const GluAt<T> &at, int left)
{
    GluBeside<T> r = {};
    if (e.q.codes) {
        Codes8 c;
        load_raw(at.cg, left, c);
        __builtin_memcpy(r.g, &c, sizeof c);
        load_raw(at.cu, left, c);
        __builtin_memcpy(r.u, &c, sizeof c);
        r.sg = left > 0 ? *at.sg : 0.f;
        r.su = left > 0 ? *at.su : 0.f;
    } else {
        Raw8<T> v;
        load_raw(at.z, left, v);
        __builtin_memcpy(r.g, &v, sizeof v);
        load_raw(at.z + F, left, v);
        __builtin_memcpy(r.u, &v, sizeof v);
    }
    b = r;
}
template <typename T>
__device__ __forceinline__ void kept_values(const uint32_t (&w)[GluBeside<T>::W], bool codes, float scale, float (&v)[8])
{
    Codes8 c;
    Raw8<T> r;
    __builtin_memcpy(&c, w, sizeof c);
    __builtin_memcpy(&r, w, sizeof r);
    if (codes) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = code_value(c.at(i), scale);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = r.at(i);
    }
}
template <typename T>
__device__ __forceinline__ void glu_gate_epilogue(const Epi &e, int F, const float (&v)[8], const GluBeside<T> &b,
                                                  const GluAt<T> &at, int left, float (&sg)[8], float (&su)[8])
{
    float g[8], u[8], a[8], s[8];
    kept_values<T>(b.g, e.q.codes != nullptr, b.sg, g);
    kept_values<T>(b.u, e.q.codes != nullptr, b.su, u);
    act_both<T>(g, e.act, a, s);
    if (e.hidden) {
        float h[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            h[i] = a[i] * u[i];
        store8(at.h, left, h);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        s[i] *= v[i] * u[i];
        a[i] *= v[i];
    }
    if (e.sums)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            sg[i] += i < left ? s[i] : 0.f;
            su[i] += i < left ? a[i] : 0.f;
        }
    store8(at.y, left, s);
    store8(at.y + F, left, a);
}

// A wave's accumulators of 16 NA rows by 64 hidden columns through the gated
// epilogue: fragments 0 .. 3 of a row hold g, 4 .. 7 u.  Alone, eight lanes take
// a row, eight rows a step (no checkpoint then).  PAIR: two waves hold the 128
// columns of a group, in neighbouring parts of LDS, and each takes half of the
// rows whole, sixteen lanes a row.  WHOLE: its columns all exist.
template <typename T, int NA, bool PAIR, bool WHOLE>
__device__ __forceinline__ void put_glu_rows(const Gemm &g, const char *lds, int64_t m0, int n0, int wn)
{
    constexpr int L = PAIR ? 16 : 8, STEP = 64 / L, ROWS = PAIR ? NA * 8 : NA * 16;
    const int lane = threadIdx.x & 63, place = lane % L;
    const int n = n0 - (PAIR ? wn * 64 : 0) + place * 8, c = (place & 7) * 2;
    const int cols = WHOLE ? 8 : g.N - n;
    const int first = PAIR ? wn * ROWS : 0;
    if (PAIR)
        lds += (place / 8 - wn) * NA * 8192;
    float bg[8], bu[8];
    glu_bias<T>(g.e, g.N, n, bg, bu);
    GluAt<T> at(g.e, m0 + first + lane / L, n);
#pragma unroll 1
    for (int r0 = 0; r0 < ROWS; r0 += STEP, at.step(g.e, STEP)) {
        const int row = first + r0 + lane / L;
        const auto chunk = [&](int k) { return *reinterpret_cast<const f32x4 *>(lds + row * 512 + (k ^ (row & 31)) * 16); };
        const f32x4 g0 = chunk(c), g1 = chunk(c + 1), u0 = chunk(16 + c), u1 = chunk(17 + c);
        float vg[8] = {g0[0], g0[1], g0[2], g0[3], g1[0], g1[1], g1[2], g1[3]};
        float vu[8] = {u0[0], u0[1], u0[2], u0[3], u1[0], u1[1], u1[2], u1[3]};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            vg[i] += bg[i];
            vu[i] += bu[i];
        }
        glu_epilogue<T, PAIR, WHOLE>(g.e, g.N, vg, vu, at, n, m0 + row < g.M ? cols : 0);
    }
}
template <typename T, int NA>
__device__ __forceinline__ void put_glu_gate_rows(const Gemm &g, const char *lds, int64_t m0, int n0, int end, float (&sg)[8],
                                                  float (&su)[8])
{
    const int lane = threadIdx.x & 63, n = n0 + (lane & 15) * 8, c = (lane & 15) * 2;
    const int cols = end - n;
    GluAt<T> at(g.e, m0 + (lane >> 4), n);
#pragma unroll 1
    for (int r0 = 0; r0 < NA * 4; r0 += 4) {
        GluBeside<T> beside[4];
        const auto left = [&](int u) { return m0 + (r0 + u) * 4 + (lane >> 4) < g.M ? cols : 0; };
        GluAt<T> ahead = at;
#pragma unroll
        for (int u = 0; u < 4; ++u, ahead.step(g.e, 4))
            load_glu_beside<T>(g.e, g.N, beside[u], ahead, left(u));
#pragma unroll
        for (int u = 0; u < 4; ++u, at.step(g.e, 4)) {
            const int row = (r0 + u) * 4 + (lane >> 4);
            const f32x4 lo = *reinterpret_cast<const f32x4 *>(lds + row * 512 + (c ^ (row & 31)) * 16);
            const f32x4 hi = *reinterpret_cast<const f32x4 *>(lds + row * 512 + ((c + 1) ^ (row & 31)) * 16);
            const float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
            glu_gate_epilogue<T>(g.e, g.N, v, beside[u], at, left(u), sg, su);
        }
    }
}

// The workgroup's waves meet with their LDS accesses done; what they still have
// to store goes on (a barrier with a fence waits for it).
__device__ __forceinline__ void lds_meet()
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// The tile's columns stop at `end`.  `part`: the piece's rows and columns of
// this wave, ld a row, or nullptr.  wn: the wave's place along
// the columns; sg, su: see glu_gate_epilogue.
template <typename T, int KIND, int NA, int WN>
__device__ __forceinline__ void put_tile(const Gemm &g, const f32x4 (&acc)[NA][8], char *lds, int64_t m0, int n0,
                                         int end, float *part, int ld, int wn, float (&sg)[8], float (&su)[8])
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
    if constexpr (KIND == kGluForward && WN == 2)
        if (g.e.q.codes) {
            lds_meet();
            if (n0 - wn * 64 + 128 <= g.N)
                put_glu_rows<T, NA, true, true>(g, lds, m0, n0, wn);
            else
                put_glu_rows<T, NA, true, false>(g, lds, m0, n0, wn);
            lds_meet();   // before the parts are written again
            return;
        }
    // the wave reads what its own lanes wrote: LDS keeps a wave's order
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    if constexpr (KIND == kGluForward)
        put_glu_rows<T, NA, false, false>(g, lds, m0, n0, wn);
    else if constexpr (KIND == kGluGate)
        put_glu_gate_rows<T, NA>(g, lds, m0, n0, end, sg, su);
    else if (n0 + 128 <= end)
        put_rows<T, KIND, NA, true>(g, lds, m0, n0, end);
    else
        put_rows<T, KIND, NA, false>(g, lds, m0, n0, end);
}

// Tile `id` of the product's order: bands of four rows of tiles, column by
// column, so that what an XCD's CUs read together stays in its L2.  A launch has
// under 2^26 tiles.
__device__ __forceinline__ void tile_at(const Gemm &g, uint32_t id, int &tile_m, int &tile_n)
{
    const uint32_t wide = 4u * g.tn, band = id / wide, in = id - band * wide, height = min(g.tm - band * 4, 4u);
    const uint32_t col = height == 4 ? in / 4 : in / height;
    tile_m = static_cast<int>(band * 4 + in - col * height);
    tile_n = static_cast<int>(col);
}

}  // namespace acsc
