// Layer norm of token rows: forward (optionally writing the 8-bit checkpoint
// of its input), the output again from kept statistics, and backward with the
// reduction of the weight gradients over the rows.
//
// All of it is HBM bound: a row is read once into registers (eight columns a
// lane and chunk), its statistics are taken there (the variance from centred
// values), and the result is written.  NT threads share a row, in chunks of
// 8 NT columns; rows of up to 2048 columns belong to one wave, which needs no
// barrier, wider ones to a workgroup.
#include "rows.h"

#include <type_traits>

namespace acsc {
namespace {

constexpr int kMaxH = 32768;

template <typename T>
struct Fwd {
    const T *x;
    int64_t ldx;
    Q8 src;                     // recompute from a checkpoint
    const T *gamma, *beta;
    T *y;
    int64_t ldy;
    float *mean, *rstd;         // out (forward) or in (recompute)
    Q8 q;                       // checkpoint out
    int64_t rows;
    int H;
    float eps;
};

// NT threads a row; workgroups of max(NT, 256) threads.
template <typename T, int NT, int CH, bool AGAIN>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void ln_forward_kernel(Fwd<T> p)
{
    constexpr int RPB = NT < 256 ? 256 / NT : 1;
    __shared__ float slots[2][NT / 64];
    const int t = threadIdx.x % NT;
    const int64_t row = (blockIdx.y * static_cast<int64_t>(gridDim.x) + blockIdx.x) * RPB +
                        (RPB > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / NT) : 0);
    if (row >= p.rows)
        return;
    float v[CH][8];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (c * NT + t) * 8;
        if (AGAIN && p.src.codes)
            load_codes(p.src.codes + row * p.src.ldc + col, p.H - col,
                       col < p.H ? p.src.scales[row * p.src.lds + col / kGroup] : 0.f, v[c]);
        else
            load8(p.x + row * p.ldx + col, p.H - col, v[c]);
    }
    float mu, rs;
    if (AGAIN) {
        mu = p.mean[row];
        rs = p.rstd[row];
    } else {
        float s[1] = {0.f};
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                s[0] += v[c][i];
        row_sum<NT>(s, slots[0]);
        mu = s[0] / p.H;
        s[0] = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int left = p.H - (c * NT + t) * 8;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = i < left ? v[c][i] - mu : 0.f;
                s[0] += d * d;
            }
        }
        row_sum<NT>(s, slots[1]);
        rs = 1.f / sqrtf(s[0] / p.H + p.eps);
        if (t == 0) {
            if (p.mean)
                p.mean[row] = mu;
            if (p.rstd)
                p.rstd[row] = rs;
        }
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (c * NT + t) * 8, left = p.H - col;
        if (!AGAIN && p.q.codes) {
            uint32_t a = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                a = max(a, mag(v[c][i]));
            a = max16(a);
            float scale, inv;
            group_scale(a, scale, inv);
            if (left > 0) {
                store_codes(p.q.codes + row * p.q.ldc + col, left, inv, v[c]);
                if ((t & 15) == 0)
                    p.q.scales[row * p.q.lds + col / kGroup] = scale;
            }
        }
        if (left > 0) {
            float g[8], b[8], o[8];
            if (p.gamma)
                load8(p.gamma + col, left, g);
            if (p.beta)
                load8(p.beta + col, left, b);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                // one rounding each, so that both forms of the kernel give the same bits
                o[i] = (v[c][i] - mu) * rs;
                o[i] = __builtin_fmaf(o[i], p.gamma ? g[i] : 1.f, p.beta ? b[i] : 0.f);
            }
            store8(p.y + row * p.ldy + col, left, o);
        }
    }
}

template <typename T>
struct Bwd {
    const T *dy;
    int64_t lddy;
    const T *x;
    int64_t ldx;
    Q8 q;
    const float *mean, *rstd;
    const T *gamma;
    const T *add;
    int64_t ldadd;
    T *dx;
    int64_t lddx;
    float *part;                // [workgroups][2][H] or nullptr
    int64_t rows;
    int H;
};

// A workgroup walks rows blockIdx.x, + gridDim.x, ... (four at a time where a
// wave holds a row) and keeps the column sums of dy h and dy in registers;
// its waves' sums meet in LDS in wave order, and every workgroup leaves one
// partial.  The next row's loads leave before a row is worked on: 16384 x
// 2048 in 54 us, its 268 MB at 5.0 TB/s (131 without).  KEPT: the row comes
// from its checkpoint.  SUMS: rows past 16384 columns leave no registers for
// the sums (4096 x 28672 with them: 940 us, most of it spilled registers);
// ln_sums_kernel takes those in a pass of its own.
template <typename T, int NT, int CH, bool KEPT, bool SUMS>
__global__ __launch_bounds__(NT < 256 ? 256 : NT, NT <= 256 ? 2 : 1) void ln_backward_kernel(Bwd<T> p)
{
    constexpr int RPB = NT < 256 ? 256 / NT : 1;
    __shared__ float slots[2][2 * (NT / 64)];
    __shared__ float meet[RPB > 1 ? 2 * NT * CH * 8 : 1];
    const int t = threadIdx.x % NT;
    const int sub = RPB > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / NT) : 0;
    float dg[CH][8], db[CH][8];
    Raw8<T> w[CH];
    const auto load_gamma = [&]() {
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if (p.gamma)
                load_raw(p.gamma + (c * NT + t) * 8, p.H - (c * NT + t) * 8, w[c]);
    };
    if (SUMS)
        load_gamma();
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            dg[c][i] = db[c][i] = 0.f;
    // a row as it is stored
    struct Row {
        typename std::conditional<KEPT, Codes8, Raw8<T>>::type x[CH];
        Raw8<T> dy[CH];
        float scale[CH], mu, rs;
    };
    const auto load = [&](Row &r, int64_t row) {
        r.mu = p.mean[row];
        r.rs = p.rstd[row];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (c * NT + t) * 8, left = p.H - col;
            if constexpr (KEPT) {
                load_raw(p.q.codes + row * p.q.ldc + col, left, r.x[c]);
                r.scale[c] = left > 0 ? p.q.scales[row * p.q.lds + col / kGroup] : 0.f;
            } else {
                load_raw(p.x + row * p.ldx + col, left, r.x[c]);
            }
            load_raw(p.dy + row * p.lddy + col, left, r.dy[c]);
        }
    };
    int flip = 0;
    const int64_t stride = static_cast<int64_t>(gridDim.x) * RPB, first = static_cast<int64_t>(blockIdx.x) * RPB + sub;
    Row cur, next;
    if (SUMS && first < p.rows)
        load(next, first);
    for (int64_t row = first; row < p.rows; row += stride, flip ^= 1) {
        Raw8<T> add[CH];
        if (SUMS)
            cur = next;
        else
            load(cur, row);
        if (p.add)
#pragma unroll
            for (int c = 0; c < CH; ++c)
                load_raw(p.add + row * p.ldadd + (c * NT + t) * 8, p.H - (c * NT + t) * 8, add[c]);
        if (SUMS && row + stride < p.rows)
            load(next, row + stride);
        if (!SUMS)
            load_gamma();
        const auto h = [&](int c, int i) {
            return ((KEPT ? code_value(cur.x[c].at(i), cur.scale[c]) : cur.x[c].at(i)) - cur.mu) * cur.rs;
        };
        const auto g = [&](int c, int i) { return p.gamma ? cur.dy[c].at(i) * w[c].at(i) : cur.dy[c].at(i); };
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            again(w[c].w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                // past the end of the row dy = 0, which leaves every sum alone
                const float hi = h(c, i), dy = cur.dy[c].at(i), gi = g(c, i);
                if (SUMS) {
                    dg[c][i] += dy * hi;
                    db[c][i] += dy;
                }
                s[0] += gi;
                s[1] += gi * hi;
            }
        }
        row_sum<NT>(s, slots[flip]);
        const float m1 = s[0] / p.H, m2 = s[1] / p.H;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (c * NT + t) * 8, left = p.H - col;
            again(cur.x[c].w);
            again(cur.dy[c].w);
            again(w[c].w);
            if (left > 0) {
                float o[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    o[i] = cur.rs * (g(c, i) - m1 - h(c, i) * m2);
                    if (p.add)
                        o[i] += add[c].at(i);
                }
                store8(p.dx + row * p.lddx + col, left, o);
            }
        }
    }
    if (!SUMS || !p.part)
        return;
    if (RPB > 1) {
        for (int v = 0; v < RPB; ++v) {
            if (sub == v) {
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        // [sum][chunk][i][lane]: consecutive lanes in consecutive banks
                        float *m = meet + ((c * 8 + i) * NT + t);
                        m[0] = v ? m[0] + dg[c][i] : dg[c][i];
                        m[NT * CH * 8] = v ? m[NT * CH * 8] + db[c][i] : db[c][i];
                    }
            }
            __syncthreads();
        }
        if (sub != 0)
            return;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                dg[c][i] = meet[(c * 8 + i) * NT + t];
                db[c][i] = meet[(c * 8 + i) * NT + t + NT * CH * 8];
            }
    }
    float *out = p.part + static_cast<int64_t>(blockIdx.x) * 2 * p.H;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (c * NT + t) * 8, left = p.H - col;
        if (left > 0) {
            store8(out + col, left, dg[c]);
            store8(out + p.H + col, left, db[c]);
        }
    }
}

// dx of fp32 rows past 8192 columns, which with their sums leave no registers
// either: a workgroup reads a row for its two sums and again, from the caches,
// for dx, with the column sums taken by ln_sums_kernel (8192 x 28672: 1185 us;
// held in registers, 1024 threads, with 300 bytes a lane of them spilled: 2540).
template <bool KEPT>
__global__ __launch_bounds__(1024, 8) void ln_backward_wide_kernel(Bwd<float> p)
{
    __shared__ float slots[2][32];
    int flip = 0;
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x, flip ^= 1) {
        const float mu = p.mean[row], rs = p.rstd[row];
        // eight columns: dy gamma and the normalised input
        const auto load = [&](int col, float (&g)[8], float (&h)[8]) {
            const int left = p.H - col;
            float w[8];
            if (KEPT)
                load_codes(p.q.codes + row * p.q.ldc + col, left, p.q.scales[row * p.q.lds + col / kGroup], h);
            else
                load8(p.x + row * p.ldx + col, left, h);
            load8(p.dy + row * p.lddy + col, left, g);
            if (p.gamma)
                load8(p.gamma + col, left, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                h[i] = (h[i] - mu) * rs;
                g[i] = p.gamma ? g[i] * w[i] : g[i];
            }
        };
        float s[2] = {0.f, 0.f};
#pragma unroll 1
        for (int col = threadIdx.x * 8; col < p.H; col += 8192) {
            float g[8], h[8];
            load(col, g, h);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                s[0] += g[i];
                s[1] += g[i] * h[i];   // past the end of the row g = 0
            }
        }
        row_sum<1024>(s, slots[flip]);
        const float m1 = s[0] / p.H, m2 = s[1] / p.H;
#pragma unroll 1
        for (int col = threadIdx.x * 8; col < p.H; col += 8192) {
            const int left = p.H - col;
            float g[8], h[8], o[8];
            load(col, g, h);
            if (p.add)
                load8(p.add + row * p.ldadd + col, left, o);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = rs * (g[i] - m1 - h[i] * m2);
                o[i] = p.add ? d + o[i] : d;
            }
            store8(p.dx + row * p.lddx + col, left, o);
        }
    }
}

// The column sums of wide rows: 512 columns and one slice of the rows a
// workgroup, whose four waves take every fourth row and meet in LDS in order.
template <typename T, bool KEPT>
__global__ __launch_bounds__(256) void ln_sums_kernel(Bwd<T> p, int per)
{
    __shared__ float meet[4][2][512];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, col = blockIdx.x * 512 + lane * 8, left = p.H - col;
    const int64_t end = min<int64_t>(p.rows, (blockIdx.y + static_cast<int64_t>(1)) * per);
    float dg[8] = {}, db[8] = {};
#pragma unroll 4
    for (int64_t row = blockIdx.y * static_cast<int64_t>(per) + wave; row < end; row += 4) {
        float x[8], dy[8];
        if (KEPT)
            load_codes(p.q.codes + row * p.q.ldc + col, left, left > 0 ? p.q.scales[row * p.q.lds + col / kGroup] : 0.f, x);
        else
            load8(p.x + row * p.ldx + col, left, x);
        load8(p.dy + row * p.lddy + col, left, dy);
        const float mu = p.mean[row], rs = p.rstd[row];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            dg[i] += dy[i] * ((x[i] - mu) * rs);
            db[i] += dy[i];
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        meet[wave][0][i * 64 + lane] = dg[i];
        meet[wave][1][i * 64 + lane] = db[i];
    }
    __syncthreads();
    for (int c = threadIdx.x; c < 1024; c += 256) {
        const int which = c >> 9, k = c & 511, at = (k & 7) * 64 + (k >> 3), n = blockIdx.x * 512 + k;
        if (n < p.H)
            p.part[(static_cast<int64_t>(blockIdx.y) * 2 + which) * p.H + n] =
                ((meet[0][which][at] + meet[1][which][at]) + meet[2][which][at]) + meet[3][which][at];
    }
}

// Column sums over the partials: 64 columns and 16 slices of the partials a
// workgroup, each slice in order, the slices joined in order.  (Four slices
// left a lane 128 dependent loads: 40 us for 512 partials of 2048 columns.)
constexpr int kSlices = 16;
__global__ __launch_bounds__(64 * kSlices) void ln_join_kernel(const float *part, int n, int H, float *dgamma, float *dbeta,
                                                               int accumulate)
{
    __shared__ float meet[kSlices][64];
    const int lane = threadIdx.x & 63, sl = threadIdx.x >> 6;
    const int col = blockIdx.x * 64 + lane;       // over 2 H: the dgamma columns, then dbeta's
    const int per = (n + kSlices - 1) / kSlices, end = min(n, (sl + 1) * per);
    float s = 0.f;
    if (col < 2 * H)
#pragma unroll 8
        for (int i = sl * per; i < end; ++i)
            s += part[static_cast<int64_t>(i) * 2 * H + col];
    meet[sl][lane] = s;
    __syncthreads();
    if (sl == 0 && col < 2 * H) {
        s = meet[0][lane];
#pragma unroll
        for (int i = 1; i < kSlices; ++i)
            s += meet[i][lane];
        float *out = col < H ? dgamma : dbeta;
        if (out) {
            out += col < H ? col : col - H;
            *out = accumulate ? *out + s : s;
        }
    }
}

// Threads and chunks for a row of H columns.  Forward: two chunks a thread
// where a workgroup can hold them (16384 x 8192 bf16, us: four chunks of 256
// threads 140, two of 512 112, one of 1024 120; 16384 x 2048 with its
// checkpoint: four of a wave 44, one of 256 threads 38), and of fp32, twice the
// bytes, one (16384 x 8192: two of 512 331, one of 1024 267).  Backward: four,
// which need fewer workgroups' partials, and of fp32 two, which is what its
// registers hold (16384 x 2048: four of a wave 235, one of 256 threads 79).
struct Shape {
    int nt, ch;
};
inline Shape forward_shape(int H, bool f32)
{
    if (H <= 512)
        return {64, 1};
    if (H <= 1024)
        return {64, 2};
    if (H <= 2048)
        return {256, 1};
    if (H <= 4096)
        return f32 ? Shape{512, 1} : Shape{256, 2};
    if (H <= 8192)
        return f32 ? Shape{1024, 1} : Shape{512, 2};
    if (H <= 16384)
        return {1024, 2};
    return {1024, 4};
}
inline Shape backward_shape(int H, bool f32)
{
    if (H <= 512)
        return {64, 1};
    if (H <= 1024)
        return {64, 2};
    if (H <= 2048)
        return f32 ? Shape{256, 1} : Shape{64, 4};
    if (H <= 4096)
        return {256, 2};
    if (H <= 8192)
        return f32 ? Shape{512, 2} : Shape{256, 4};
    return {512, 4};
}

// Rows past this go without sums in the pass for dx.
inline int sums_most(bool f32) { return f32 ? 8192 : 16384; }

// Workgroups of the backward pass, which is also its number of partials; for
// wide rows the slices of the sums' own pass, of at least 32 rows.
inline int bwd_groups(int64_t rows, int H, bool f32)
{
    if (H > sums_most(f32))
        return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(rows / 32, 1024 / ((H + 511) / 512))));
    const int rpb = backward_shape(H, f32).nt == 64 ? 4 : 1;
    return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>((rows + rpb - 1) / rpb, 512)));
}

inline int check_common(int64_t rows, int H, int dt)
{
    ACSC_CHECK_ARG(dt == ACSC_F32 || dt == ACSC_BF16, ACSC_EDTYPE, "unknown dtype %d", dt);
    ACSC_CHECK_ARG(rows >= 0 && rows < (1ll << 31), ACSC_EINVAL, "rows=%lld outside [0, 2^31)", (long long)rows);
    ACSC_CHECK_ARG(H >= 1 && H <= kMaxH, ACSC_EINVAL, "H=%d outside [1, %d]", H, kMaxH);
    return ACSC_OK;
}

inline int check_mat(const void *p, int64_t rows, int64_t ld, int H, int dt, const char *name)
{
    ACSC_CHECK_ARG(rows == 0 || p, ACSC_EINVAL, "null pointer %s", name);
    ACSC_CHECK_ARG(ld >= H, ACSC_EINVAL, "ld of %s is %lld < H=%d", name, (long long)ld, H);
    ACSC_CHECK_ARG(aligned(p, dtype_size(static_cast<acsc_dtype>(dt))), ACSC_EALIGN, "%s not aligned to its elements",
                   name);
    return ACSC_OK;
}

template <typename T, bool AGAIN>
int run_forward(const Fwd<T> &p, hipStream_t st)
{
    const Shape s = forward_shape(p.H, sizeof(T) == 4);
    const int64_t blocks = s.nt == 64 ? (p.rows + 3) / 4 : p.rows;
    // a grid has under 2^32 threads along x: past 2^20 workgroups it goes on along y
    const int64_t across = std::min<int64_t>(blocks, 1 << 20);
    const dim3 grid(static_cast<unsigned>(across), static_cast<unsigned>((blocks + across - 1) / across));
    const char *tag = AGAIN ? "ln_recompute" : "ln_forward";
#define ACSC_CASE(NT, CH)                                                                                       \
    if (s.nt == NT && s.ch == CH)                                                                             \
        ACSC_LAUNCH(tag, (ln_forward_kernel<T, NT, CH, AGAIN>), grid, dim3(NT < 256 ? 256 : NT), 0, st, p);
    ACSC_CASE(64, 1)
    ACSC_CASE(64, 2)
    ACSC_CASE(256, 1)
    ACSC_CASE(256, 2)
    ACSC_CASE(512, 2)
    ACSC_CASE(512, 1)
    ACSC_CASE(1024, 1)
    ACSC_CASE(1024, 2)
    ACSC_CASE(1024, 4)
#undef ACSC_CASE
    return check_launch(tag);
}

template <typename T, bool KEPT>
int run_backward(const Bwd<T> &p, int groups, hipStream_t st)
{
    constexpr bool f32 = sizeof(T) == 4;
    if (p.H > sums_most(f32)) {
        if (p.part) {
            const int per = static_cast<int>((p.rows + groups - 1) / groups);
            ACSC_LAUNCH("ln_sums", (ln_sums_kernel<T, KEPT>), dim3((p.H + 511) / 512, groups), dim3(256), 0, st, p, per);
        }
        // after the sums, which read dy: dx may take its place
        const dim3 grid(static_cast<unsigned>(std::min<int64_t>(p.rows, 1 << 20)));
        if (p.rows) {
            if constexpr (f32)
                ACSC_LAUNCH("ln_backward", (ln_backward_wide_kernel<KEPT>), grid, dim3(1024), 0, st, p);
            else
                ACSC_LAUNCH("ln_backward", (ln_backward_kernel<T, 1024, 4, KEPT, false>), grid, dim3(1024), 0, st, p);
        }
        return check_launch("ln_backward");
    }
    const Shape s = backward_shape(p.H, f32);
    const dim3 grid(groups);
#define ACSC_CASE(NT, CH)                                                                                       \
    if (s.nt == NT && s.ch == CH)                                                                             \
        ACSC_LAUNCH("ln_backward", (ln_backward_kernel<T, NT, CH, KEPT, true>), grid, dim3(NT < 256 ? 256 : NT), 0, st, p);
    ACSC_CASE(64, 1)
    ACSC_CASE(64, 2)
    ACSC_CASE(256, 2)
    if constexpr (f32) {
        ACSC_CASE(256, 1)
        ACSC_CASE(512, 2)
    } else {
        ACSC_CASE(64, 4)
        ACSC_CASE(256, 4)
        ACSC_CASE(512, 4)
    }
#undef ACSC_CASE
    return check_launch("ln_backward");
}
template <typename T>
int run_backward(const Bwd<T> &p, int groups, hipStream_t st)
{
    return p.q.codes ? run_backward<T, true>(p, groups, st) : run_backward<T, false>(p, groups, st);
}

template <typename T>
const T *as(const void *p)
{
    return static_cast<const T *>(p);
}

}  // namespace
}  // namespace acsc

using namespace acsc;

extern "C" int ln_forward(const void *x, acsc_dtype dt, int64_t rows, int H, int64_t ld_x, const void *gamma,
                          const void *beta, float eps, void *y, int64_t ld_y, float *mean, float *rstd,
                          const q8_tensor *q, hipStream_t stream)
{
    clear_error();
    if (int rc = check_common(rows, H, dt))
        return rc;
    ACSC_CHECK_ARG(std::isfinite(eps) && eps > 0.f, ACSC_EINVAL, "eps=%g must be positive", eps);
    if (int rc = check_mat(x, rows, ld_x, H, dt, "x"))
        return rc;
    if (int rc = check_mat(y, rows, ld_y, H, dt, "y"))
        return rc;
    ACSC_CHECK_ARG(y != x || rows == 0 || ld_y == ld_x, ACSC_EINVAL, "y in place of x needs ld_y == ld_x");
    ACSC_CHECK_ARG(aligned(gamma, dtype_size(dt)) && aligned(beta, dtype_size(dt)), ACSC_EALIGN,
                   "gamma or beta not aligned to its elements");
    ACSC_CHECK_ARG(aligned(mean, 4) && aligned(rstd, 4), ACSC_EALIGN, "mean or rstd not 4-byte aligned");
    if (q)
        if (int rc = check_q8(q, rows, H))
            return rc;
    if (rows == 0)
        return ACSC_OK;
    const Q8 none{nullptr, nullptr, 0, 0};
    if (dt == ACSC_BF16)
        return run_forward<uint16_t, false>({as<uint16_t>(x), ld_x, none, as<uint16_t>(gamma), as<uint16_t>(beta),
                                             static_cast<uint16_t *>(y), ld_y, mean, rstd, q8_of(q), rows, H, eps}, stream);
    return run_forward<float, false>({as<float>(x), ld_x, none, as<float>(gamma), as<float>(beta),
                                      static_cast<float *>(y), ld_y, mean, rstd, q8_of(q), rows, H, eps}, stream);
}

extern "C" int ln_recompute(const void *x, int64_t ld_x, const q8_tensor *q, acsc_dtype dt, int64_t rows, int H,
                            const float *mean, const float *rstd, const void *gamma, const void *beta, void *y,
                            int64_t ld_y, hipStream_t stream)
{
    clear_error();
    if (int rc = check_common(rows, H, dt))
        return rc;
    ACSC_CHECK_ARG(rows == 0 || (x != nullptr) != (q != nullptr), ACSC_EINVAL, "exactly one of x and its checkpoint is needed");
    if (x)
        if (int rc = check_mat(x, rows, ld_x, H, dt, "x"))
            return rc;
    if (q)
        if (int rc = check_q8(q, rows, H))
            return rc;
    if (int rc = check_mat(y, rows, ld_y, H, dt, "y"))
        return rc;
    ACSC_CHECK_ARG(y != x || rows == 0 || ld_y == ld_x, ACSC_EINVAL, "y in place of x needs ld_y == ld_x");
    ACSC_CHECK_ARG(rows == 0 || (mean && rstd), ACSC_EINVAL, "null statistics");
    ACSC_CHECK_ARG(aligned(mean, 4) && aligned(rstd, 4), ACSC_EALIGN, "mean or rstd not 4-byte aligned");
    ACSC_CHECK_ARG(aligned(gamma, dtype_size(dt)) && aligned(beta, dtype_size(dt)), ACSC_EALIGN,
                   "gamma or beta not aligned to its elements");
    if (rows == 0)
        return ACSC_OK;
    const Q8 none{nullptr, nullptr, 0, 0};
    float *mu = const_cast<float *>(mean), *rs = const_cast<float *>(rstd);   // read only there
    if (dt == ACSC_BF16)
        return run_forward<uint16_t, true>({as<uint16_t>(x), ld_x, q8_of(q), as<uint16_t>(gamma), as<uint16_t>(beta),
                                            static_cast<uint16_t *>(y), ld_y, mu, rs, none, rows, H, 0.f}, stream);
    return run_forward<float, true>({as<float>(x), ld_x, q8_of(q), as<float>(gamma), as<float>(beta),
                                     static_cast<float *>(y), ld_y, mu, rs, none, rows, H, 0.f}, stream);
}

extern "C" int ln_workspace_size(int64_t rows, int H, size_t *bytes)
{
    clear_error();
    if (int rc = check_common(rows, H, ACSC_F32))
        return rc;
    ACSC_CHECK_ARG(bytes, ACSC_EINVAL, "null pointer bytes");
    *bytes = static_cast<size_t>(std::max(bwd_groups(rows, H, false), bwd_groups(rows, H, true))) * 2 * H * sizeof(float);
    return ACSC_OK;
}

extern "C" int ln_backward(const void *dy, int64_t ld_dy, const void *x, int64_t ld_x, const q8_tensor *q,
                           acsc_dtype dt, int64_t rows, int H, const float *mean, const float *rstd,
                           const void *gamma, const void *add, int64_t ld_add, void *dx, int64_t ld_dx, float *dgamma,
                           float *dbeta, int accumulate, void *ws, size_t ws_bytes, hipStream_t stream)
{
    clear_error();
    if (int rc = check_common(rows, H, dt))
        return rc;
    ACSC_CHECK_ARG(rows == 0 || (x != nullptr) != (q != nullptr), ACSC_EINVAL, "exactly one of x and its checkpoint is needed");
    if (int rc = check_mat(dy, rows, ld_dy, H, dt, "dy"))
        return rc;
    if (x)
        if (int rc = check_mat(x, rows, ld_x, H, dt, "x"))
            return rc;
    if (q)
        if (int rc = check_q8(q, rows, H))
            return rc;
    if (add)
        if (int rc = check_mat(add, rows, ld_add, H, dt, "add"))
            return rc;
    if (int rc = check_mat(dx, rows, ld_dx, H, dt, "dx"))
        return rc;
    ACSC_CHECK_ARG(dx != dy || rows == 0 || ld_dx == ld_dy, ACSC_EINVAL, "dx in place of dy needs ld_dx == ld_dy");
    ACSC_CHECK_ARG(dx != x || rows == 0 || ld_dx == ld_x, ACSC_EINVAL, "dx in place of x needs ld_dx == ld_x");
    ACSC_CHECK_ARG(dx != add || rows == 0 || ld_dx == ld_add, ACSC_EINVAL, "dx in place of add needs ld_dx == ld_add");
    ACSC_CHECK_ARG(rows == 0 || (mean && rstd), ACSC_EINVAL, "null statistics");
    ACSC_CHECK_ARG(aligned(mean, 4) && aligned(rstd, 4) && aligned(dgamma, 4) && aligned(dbeta, 4), ACSC_EALIGN,
                   "an fp32 array is not 4-byte aligned");
    ACSC_CHECK_ARG(aligned(gamma, dtype_size(dt)), ACSC_EALIGN, "gamma not aligned to its elements");
    const bool sums = dgamma || dbeta;
    const int groups = bwd_groups(rows, H, dt == ACSC_F32);
    if (sums) {
        ACSC_CHECK_ARG(ws, ACSC_EINVAL, "null workspace");
        ACSC_CHECK_ARG(aligned(ws, 256), ACSC_EALIGN, "workspace not 256-byte aligned");
        const size_t need = static_cast<size_t>(groups) * 2 * H * sizeof(float);
        ACSC_CHECK_ARG(ws_bytes >= need, ACSC_ENOSPC, "workspace of %zu bytes, %zu needed", ws_bytes, need);
    }
    if (rows == 0 && !sums)
        return ACSC_OK;
    float *part = sums ? static_cast<float *>(ws) : nullptr;
    int rc;
    if (dt == ACSC_BF16)
        rc = run_backward<uint16_t>({as<uint16_t>(dy), ld_dy, as<uint16_t>(x), ld_x, q8_of(q), mean, rstd,
                                     as<uint16_t>(gamma), as<uint16_t>(add), ld_add, static_cast<uint16_t *>(dx), ld_dx,
                                     part, rows, H}, groups, stream);
    else
        rc = run_backward<float>({as<float>(dy), ld_dy, as<float>(x), ld_x, q8_of(q), mean, rstd, as<float>(gamma),
                                  as<float>(add), ld_add, static_cast<float *>(dx), ld_dx, part, rows, H}, groups, stream);
    if (rc || !sums)
        return rc;
    ACSC_LAUNCH("ln_join", ln_join_kernel, dim3((2 * H + 63) / 64), dim3(64 * kSlices), 0, stream, part, groups, H, dgamma, dbeta,
                accumulate);
    return check_launch("ln_join");
}
