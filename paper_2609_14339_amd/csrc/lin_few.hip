// A linear layer's forward product for few tokens (up to 16): the weights are read once, straight into the matrix cores' lanes, at
// whatever stride and alignment they have.
//
// What bounds it is the weights' bytes: no LDS, no barrier on the way.  A
// workgroup of eight waves takes 16 outputs; in each of its 16 rows of W the
// waves take the 128-byte lines in turn, four lines (eight 16-byte loads a
// lane) in flight, and multiply them with the same k of the tokens, which
// stay in the caches.  Their sums meet in LDS in wave order.  One token, bf16
// 4096 -> 14336: 24 us, 4.9 TB/s of weights, what a copy reaches.
#include "lin_plan.h"

namespace acsc {
namespace {

typedef __attribute__((__vector_size__(8 * sizeof(short)))) short bf16x8;

constexpr int kWaves = 8;

// 16 bytes of a row, the first nv elements of them, zeros after.
struct __attribute__((packed, aligned(2))) Any16 {
    uint32_t w[4];
};
template <typename T>
__device__ __forceinline__ Any16 load16(const T *p, int nv)
{
    constexpr int E = 16 / sizeof(T);
    if (nv >= E)
        return *reinterpret_cast<const Any16 *>(p);
    Any16 r = {{0, 0, 0, 0}};
#pragma unroll
    for (int i = 0; i < E; ++i)
        if (i < nv) {
            if (sizeof(T) == 2)
                r.w[i / 2] |= static_cast<uint32_t>(reinterpret_cast<const uint16_t *>(p)[i]) << (16 * (i & 1));
            else
                r.w[i] = reinterpret_cast<const uint32_t *>(p)[i];
        }
    return r;
}

// Lane L of a 16-byte chunk holds row L % 16 and E values of k from E (L / 16):
// one bf16 instruction of 32 k, or four fp32 ones of every fourth k.
template <typename T>
__device__ __forceinline__ f32x4 multiply(const Any16 &w, const Any16 &x, f32x4 acc)
{
    if (sizeof(T) == 2) {
        bf16x8 a, b;
        __builtin_memcpy(&a, &w, 16);
        __builtin_memcpy(&b, &x, 16);
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, acc, 0, 0, 0);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w.w[e]), __uint_as_float(x.w[e]), acc, 0, 0, 0);
    return acc;
}

// GLU: the gated product, of whose rows of W a workgroup takes those of eight
// hidden columns, the gate's, then the up projection's.  (16 of each, twice the
// loads in flight and half the workgroups: one token 4096 -> 14336 46 us, 42 so.)
template <typename T, bool GLU>
__global__ __launch_bounds__(kWaves * 64) void lin_few_kernel(Gemm g)
{
    constexpr int E = 16 / sizeof(T), LINE = 8 * E, U = 4;   // k of a chunk and of a line; lines in flight
    __shared__ __align__(16) float meet[kWaves][16][16];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    constexpr int COLS = GLU ? 8 : 16;
    const int n0 = blockIdx.x * COLS, split = blockIdx.y;
    const int kbeg = split * g.kchunk, kend = min(g.K, kbeg + g.kchunk);
    const int k = (lane >> 4) * E;
    const T *w = static_cast<const T *>(g.B.p) + (min(n0 + lane % COLS, g.N - 1) + (GLU && lane & 8 ? g.N : 0)) * g.B.ld;
    const T *x = static_cast<const T *>(g.A.p) + min<int64_t>(lane & 15, g.M - 1) * g.A.ld;
    f32x4 acc = {0, 0, 0, 0};

    int k0 = kbeg + wave * LINE;
    for (; k0 + ((U - 1) * kWaves + 1) * LINE <= kend; k0 += U * kWaves * LINE) {
        Any16 a[U][2], b[U][2];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int at = k0 + u * kWaves * LINE + h * 4 * E + k;
                a[u][h] = *reinterpret_cast<const Any16 *>(w + at);
            }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                b[u][h] = *reinterpret_cast<const Any16 *>(x + k0 + u * kWaves * LINE + h * 4 * E + k);
        __builtin_amdgcn_sched_barrier(0);   // all loads leave before the first product
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                acc = multiply<T>(a[u][h], b[u][h], acc);
    }
    for (; k0 < kend; k0 += kWaves * LINE)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int at = k0 + h * 4 * E + k;
            acc = multiply<T>(load16(w + at, kend - at), load16(x + at, kend - at), acc);
        }

    *reinterpret_cast<f32x4 *>(&meet[wave][lane & 15][(lane >> 4) * 4]) = acc;
    __syncthreads();
    const int m = threadIdx.x >> 1, c = (threadIdx.x & 1) * 8, n = n0 + c;   // eight sums a thread
    if (m >= 16 || m >= g.M)
        return;
    float v[8] = {};
    for (int i = 0; i < kWaves; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j)
            v[j] += meet[i][m][c + j];
    if constexpr (GLU) {
        if (g.part) {
            // the gate's threads and the up projection's
            store8(g.part + (split * g.M + m) * 2 * g.ldp + (c ? g.ldp : 0) + n0, g.N - n0, v);
            return;
        }
        float u[8], bg[8], bu[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            u[j] = __shfl_down(v[j], 1);
        if (c)
            return;
        glu_bias<T>(g.e, g.N, n0, bg, bu);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[j] += bg[j];
            u[j] += bu[j];
        }
        glu_epilogue<T, false>(g.e, g.N, v, u, GluAt<T>(g.e, m, n0), n0, g.N - n0);
        return;
    }
    if (g.part) {
        store8(g.part + (split * g.M + m) * g.ldp + n, g.N - n, v);
    } else {
        float bias[8];
        load_bias<T, kForward>(g.e, n, g.N, bias);
        Beside<T> beside;
        if (has_beside<T, kForward>(g.e))
            load_beside<T, kForward>(g.e, beside, m, n, g.N - n);
        epilogue<T, kForward>(g.e, v, bias, beside, m, n, g.N - n);   // without a checkpoint: lanes of their own
    }
}

// The weight gradient of few tokens: outer products, bound by writing dW.  A
// lane holds eight columns of the T inputs in fp32 (formed here from what was
// kept, so nothing is rounded on the way), a wave `per` rows of dW one after
// the other; dz waits in LDS.  The workgroups of the first columns add up db.
constexpr int kRowsMost = 64;
template <typename T, typename TO, int TT>
__global__ __launch_bounds__(256) void lin_few_weight_kernel(Gemm g, Kept kept, int per, float *db)
{
    __shared__ __align__(16) float dz[4 * kRowsMost][TT];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int n = blockIdx.x * 512 + lane * 8, left = g.N - n;
    const int64_t m0 = static_cast<int64_t>(blockIdx.y) * 4 * per;
    const int rows = static_cast<int>(min<int64_t>(g.M - m0, 4 * per));
    for (int i = threadIdx.x; i < rows * TT; i += 256) {
        const int t = i / rows, r = i - t * rows;
        float v = 0.f;
        if (t < g.K) {
            const T x = static_cast<const T *>(g.A.p)[t * g.A.ld + m0 + r];
            if constexpr (sizeof(T) == 2)
                v = bf16_to_f32(x);
            else
                v = x;
        }
        dz[r][t] = v;
    }
    float a[TT][8];
#pragma unroll
    for (int t = 0; t < TT; ++t) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            a[t][i] = 0.f;
        if (t < g.K) {
            if (kept.q.codes)
                load_codes(kept.q.codes + t * kept.q.ldc + n, left, left > 0 ? kept.q.scales[t * kept.q.lds + n / kGroup] : 0.f,
                           a[t]);
            else
                load8(static_cast<const T *>(g.B.p) + t * g.B.ld + n, left, a[t]);
            apply_act<float>(a[t], kept.act);
        }
    }
    __syncthreads();
    if (db && blockIdx.x == 0 && threadIdx.x < rows) {
        float s = 0.f;
        for (int t = 0; t < g.K; ++t)
            s += dz[threadIdx.x][t];
        db[m0 + threadIdx.x] = g.e.accumulate ? db[m0 + threadIdx.x] + s : s;
    }
    const int end = min(rows, (wave + 1) * per);
    for (int r = wave * per; r < end; ++r) {
        float v[8] = {};
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            const float d = dz[r][t];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                v[i] = __builtin_fmaf(d, a[t][i], v[i]);
        }
        const float bias[8] = {};
        Beside<TO> beside;
        if (has_beside<TO, kWeight>(g.e))
            load_beside<TO, kWeight>(g.e, beside, m0 + r, n, left);
        epilogue<TO, kWeight>(g.e, v, bias, beside, m0 + r, n, left);
    }
}

template <typename T, typename TO>
void launch_weight(const Gemm &g, const Kept &kept, float *db, hipStream_t st, const char *tag)
{
    const int64_t cols = (g.N + 511) / 512;
    // rows of a wave: two workgroups a CU, at most 64 to an activation
    const int per = static_cast<int>(std::max<int64_t>(2, std::min<int64_t>(kRowsMost, g.M * cols / (4 * 512))));
    const dim3 grid(static_cast<unsigned>(cols), static_cast<unsigned>((g.M + 4 * per - 1) / (4 * per)));
    if (g.K <= 4)
        ACSC_LAUNCH(tag, (lin_few_weight_kernel<T, TO, 4>), grid, dim3(256), 0, st, g, kept, per, db);
    else
        ACSC_LAUNCH(tag, (lin_few_weight_kernel<T, TO, 8>), grid, dim3(256), 0, st, g, kept, per, db);
}

}  // namespace

int lin_few_run(const Gemm &g, acsc_dtype dt, hipStream_t st, const char *tag)
{
    const dim3 grid(static_cast<unsigned>((g.N + 15) / 16), g.splits);
    if (dt == ACSC_BF16)
        ACSC_LAUNCH(tag, (lin_few_kernel<uint16_t, false>), grid, dim3(kWaves * 64), 0, st, g);
    else
        ACSC_LAUNCH(tag, (lin_few_kernel<float, false>), grid, dim3(kWaves * 64), 0, st, g);
    return check_launch(tag);
}

int glu_few_run(const Gemm &g, acsc_dtype dt, hipStream_t st, const char *tag)
{
    const dim3 grid(static_cast<unsigned>((g.N + 7) / 8), g.splits);
    if (dt == ACSC_BF16)
        ACSC_LAUNCH(tag, (lin_few_kernel<uint16_t, true>), grid, dim3(kWaves * 64), 0, st, g);
    else
        ACSC_LAUNCH(tag, (lin_few_kernel<float, true>), grid, dim3(kWaves * 64), 0, st, g);
    return check_launch(tag);
}

int lin_few_weight_run(const Gemm &g, const Kept &kept, acsc_dtype dt, acsc_dtype out, float *db, hipStream_t st,
                       const char *tag)
{
    if (dt == ACSC_BF16)
        out == ACSC_BF16 ? launch_weight<uint16_t, uint16_t>(g, kept, db, st, tag)
                         : launch_weight<uint16_t, float>(g, kept, db, st, tag);
    else
        out == ACSC_BF16 ? launch_weight<float, uint16_t>(g, kept, db, st, tag)
                         : launch_weight<float, float>(g, kept, db, st, tag);
    return check_launch(tag);
}

}  // namespace acsc
