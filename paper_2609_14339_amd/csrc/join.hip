// Root-mean-square norms of token rows, alone and joined with what stands
// between two blocks: the norm after a block, its gate, dropout, the scaled
// residual, and the norm before the next block.
//
//   t = b rho1 post (rho1 = 1 / sqrt(mean b^2 + eps)), or b
//   out = scale r + D(gate t)
//   y = out rho2 pre (rho2 = 1 / sqrt(mean out^2 + eps))
//
// All of it is HBM bound: r and b are read once into registers (eight columns a
// lane and chunk), out and y written once.  NT threads share a row, in chunks
// of 8 NT columns, as in the layer norm.  16384 x 8192 bf16 forward 207 us, 5.2
// TB/s; gradients of 16384 x 4096 167, 4.8 TB/s.
#include "drop.h"
#include "rows.h"

#include <atomic>
#include <type_traits>

namespace acsc {
namespace {

constexpr int kMaxH = 32768;
typedef float f32x4 __attribute__((ext_vector_type(4)));

template <typename T>
struct Fwd {
    const T *r;                  // the norm's own input where there is no b
    int64_t ldr;
    const T *b;                  // nullptr: the norm alone
    int64_t ldb;
    Q8 src;                      // again: the input's checkpoint
    const T *post, *gate, *pre;
    T *out;
    int64_t ldo;
    T *y;                        // nullptr: no norm after
    int64_t ldy;
    float *rstd_post, *rstd_pre;
    Q8 q_out, q_b;
    Drop drop;
    int64_t rows;
    int H;
    float scale, eps;
};

// The codes of eight values of a row, whose group lies on sixteen lanes.
__device__ __forceinline__ void put_codes(const Q8 &q, int64_t row, int col, int left, const float (&v)[8])
{
    uint32_t a = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        a = max(a, mag(v[i]));
    a = max16(a);
    float scale, inv;
    group_scale(a, scale, inv);
    if (left > 0) {
        store_codes(q.codes + row * q.ldc + col, left, inv, v);
        if (col % kGroup == 0)
            q.scales[row * q.lds + col / kGroup] = scale;
    }
}

// Zeros in the place of values past a row's end, which a norm's NaN (0 rho) has
// made NaN: they share sums and groups with values that exist, of which the mask
// may have kept none (without one the row is NaN throughout).
__device__ __forceinline__ void clear_past(float (&v)[8], int left)
{
    if (left < 8)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = i < left ? v[i] : 0.f;
}

// NT threads a row; workgroups of max(NT, 256) threads.  JOIN: with a branch b;
// AGAIN: y from a kept rho2.  y is taken from out before it is rounded.
template <typename T, int NT, int CH, bool JOIN, bool AGAIN>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void join_forward_kernel(Fwd<T> p)
{
    constexpr int RPB = NT < 256 ? 256 / NT : 1;
    __shared__ float slots[2][NT / 64];
    const int t = threadIdx.x % NT;
    const int64_t row = (blockIdx.y * static_cast<int64_t>(gridDim.x) + blockIdx.x) * RPB +
                        (RPB > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / NT) : 0);
    if (row >= p.rows)
        return;
    float v[CH][8];
    Raw8<T> r[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (c * NT + t) * 8;
        if (AGAIN && p.src.codes)
            load_codes(p.src.codes + row * p.src.ldc + col, p.H - col,
                       col < p.H ? p.src.scales[row * p.src.lds + col / kGroup] : 0.f, v[c]);
        else if (JOIN)
            load8(p.b + row * p.ldb + col, p.H - col, v[c]);
        else
            load8(p.r + row * p.ldr + col, p.H - col, v[c]);
    }
    if (JOIN) {
#pragma unroll
        for (int c = 0; c < CH; ++c)
            load_raw(p.r + row * p.ldr + (c * NT + t) * 8, p.H - (c * NT + t) * 8, r[c]);
        float rs = 1.f;
        if (p.post) {
            float s[1] = {0.f};
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    s[0] += v[c][i] * v[c][i];
            row_sum<NT>(s, slots[0]);
            rs = 1.f / sqrtf(s[0] / p.H + p.eps);
            if (t == 0 && p.rstd_post)
                p.rstd_post[row] = rs;
        }
        const DropRow d = drop_row(p.drop, row);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (c * NT + t) * 8, left = p.H - col;
            if (p.q_b.codes)
                put_codes(p.q_b, row, col, left, v[c]);
            float w[8];
            if (p.post) {
                load8(p.post + col, left, w);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    v[c][i] = v[c][i] * rs * w[i];
            }
            if (p.gate) {
                load8(p.gate + col, left, w);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    v[c][i] *= w[i];
            }
            if (p.drop.below) {
                drop8(p.drop, d, col, v[c]);
                clear_past(v[c], left);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
                v[c][i] = __builtin_fmaf(p.scale, r[c].at(i), v[c][i]);
            if (left > 0)
                store8(p.out + row * p.ldo + col, left, v[c]);
        }
    }
    if (JOIN && !p.y && !p.q_out.codes)
        return;
    float rs = 0.f;
    if (AGAIN) {
        rs = p.rstd_pre[row];
    } else if (p.y) {
        float s[1] = {0.f};
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                s[0] += v[c][i] * v[c][i];   // zeros past the end of the row
        row_sum<NT>(s, slots[1]);
        rs = 1.f / sqrtf(s[0] / p.H + p.eps);
        if (t == 0 && p.rstd_pre)
            p.rstd_pre[row] = rs;
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (c * NT + t) * 8, left = p.H - col;
        if (!AGAIN && p.q_out.codes)
            put_codes(p.q_out, row, col, left, v[c]);
        if (left > 0 && p.y) {
            float w[8], o[8];
            if (p.pre)
                load8(p.pre + col, left, w);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                o[i] = v[c][i] * rs * (p.pre ? w[i] : 1.f);
            store8(p.y + row * p.ldy + col, left, o);
        }
    }
}

template <typename T>
struct Bwd {
    const T *dout;               // or nullptr
    int64_t lddo;
    const T *dy;                 // nullptr: no norm after
    int64_t lddy;
    const T *out;                // the norm's input, or its checkpoint
    int64_t ldo;
    Q8 q_out;
    const T *b;
    int64_t ldb;
    Q8 q_b;
    const T *post, *gate, *pre;
    const float *rstd_post, *rstd_pre;
    T *dr;                       // or nullptr
    int64_t lddr;
    T *db;                       // nullptr: the norm alone
    int64_t lddb;
    float *part;                 // [workgroups][2][H] or nullptr: sums of dy h2, and of D(t) h1
    Drop drop;
    int64_t rows;
    int H;
    float scale;
};

// One row's values of eight columns, loaded where the formula has them.
template <typename T, bool KEPT>
struct Src {
    typename std::conditional<KEPT, Codes8, Raw8<T>>::type x;
    float scale;
    __device__ __forceinline__ void load(const T *p, int64_t ld, const Q8 &q, int64_t row, int col, int left)
    {
        if constexpr (KEPT) {
            load_raw(q.codes + row * q.ldc + col, left, x);
            scale = left > 0 ? q.scales[row * q.lds + col / kGroup] : 0.f;
        } else {
            load_raw(p + row * ld + col, left, x);
        }
    }
    __device__ __forceinline__ float at(int i) const { return KEPT ? code_value(x.at(i), scale) : x.at(i); }
};

// With t the whole gradient of out and u = D(t) (the same mask):
//   h2 = out rho2, g = dy pre, t = dout + rho2 (g - h2 mean(g h2)), dr = scale t
//   h1 = b rho1 (or b), e = u gate post, db = rho1 (e - h1 mean(e h1)) (or e)
//   dpre = sum of dy h2,   s = sum of u h1, dgate = s post, dpost = s gate
// A workgroup walks rows blockIdx.x, + gridDim.x, ... (four at a time where a
// wave holds a row) and keeps both column sums in registers; its waves' sums
// meet in LDS in wave order, and every workgroup leaves one partial.  The gains
// stay in registers, and, AHEAD, the next row's loads leave before a row is
// worked on (16384 x 4096 bf16 167 us; 233 without either).  Sums of a row's
// terms and of columns are fp32; dr and db are rounded once, from t.
template <typename T, int NT, int CH, bool JOIN, bool KEPT, bool AHEAD>
__global__ __launch_bounds__(NT < 256 ? 256 : NT, NT <= 256 ? 2 : 1) void join_backward_kernel(Bwd<T> p)
{
    constexpr int RPB = NT < 256 ? 256 / NT : 1;
    __shared__ float slots[2][2][NT / 64];
    __shared__ float meet[RPB > 1 ? 2 * NT * CH * 8 : 1];
    const int t = threadIdx.x % NT;
    const int sub = RPB > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / NT) : 0;
    const bool branch = JOIN && (p.post || p.gate);     // whether the formula reads b
    // one chunk leaves room for what two form again from the stored words (21834 x
    // 64 bf16 29.5 us, formed again 33.6), but in the 128 registers of 1024 threads
    const auto keep = [](auto &w) {
        if (CH > 1 || !AHEAD)
            again(w);
    };
    float s2[CH][8], s1[CH][8];
    Raw8<T> pre[CH], post[CH], gate[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (c * NT + t) * 8, left = p.H - col;
        if (p.pre)
            load_raw(p.pre + col, left, pre[c]);
        if (JOIN && p.post)
            load_raw(p.post + col, left, post[c]);
        if (JOIN && p.gate)
            load_raw(p.gate + col, left, gate[c]);
    }
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            s2[c][i] = s1[c][i] = 0.f;
    // a row as it is stored
    struct Row {
        Raw8<T> dout[CH], dy[CH];
        Src<T, KEPT> x[CH], b[CH];
        float pre, post;
    };
    const auto load = [&](Row &r, int64_t row) {
        r.pre = p.dy ? p.rstd_pre[row] : 0.f;
        r.post = JOIN && p.post ? p.rstd_post[row] : 1.f;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (c * NT + t) * 8, left = p.H - col;
            if (p.dy) {
                r.x[c].load(p.out, p.ldo, p.q_out, row, col, left);
                load_raw(p.dy + row * p.lddy + col, left, r.dy[c]);
            }
            load_raw(p.dout + row * p.lddo + col, p.dout ? left : 0, r.dout[c]);
            if (branch)
                r.b[c].load(p.b, p.ldb, p.q_b, row, col, left);
        }
    };
    int flip = 0;
    const int64_t stride = static_cast<int64_t>(gridDim.x) * RPB, first = static_cast<int64_t>(blockIdx.x) * RPB + sub;
    Row cur, next;
    if (AHEAD && first < p.rows)
        load(next, first);
    for (int64_t row = first; row < p.rows; row += stride, flip ^= 1) {
        if (AHEAD) {
            cur = next;
            if (row + stride < p.rows)
                load(next, row + stride);
        } else {
            load(cur, row);
        }
        float v[CH][8];
        if (p.dy) {
            const float rs = cur.pre;
            float s[1] = {0.f};
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                keep(pre[c].w);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float h = cur.x[c].at(i) * rs, d = cur.dy[c].at(i), g = p.pre ? d * pre[c].at(i) : d;
                    s2[c][i] += d * h;       // past the end of the row dy = 0
                    s[0] += g * h;
                }
            }
            row_sum<NT>(s, slots[flip][0]);
            const float m = s[0] / p.H;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                keep(cur.x[c].x.w);
                keep(cur.dy[c].w);
                keep(pre[c].w);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float h = cur.x[c].at(i) * rs, d = cur.dy[c].at(i), g = p.pre ? d * pre[c].at(i) : d;
                    v[c][i] = cur.dout[c].at(i) + rs * (g - h * m);
                }
            }
        } else {
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    v[c][i] = cur.dout[c].at(i);
        }
        if (p.dr)
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int col = (c * NT + t) * 8, left = p.H - col;
                float o[8];
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    o[i] = JOIN ? p.scale * v[c][i] : v[c][i];
                if (left > 0)
                    store8(p.dr + row * p.lddr + col, left, o);
            }
        if (!JOIN)
            continue;
        if (p.drop.below) {
            const DropRow d = drop_row(p.drop, row);
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                drop8(p.drop, d, (c * NT + t) * 8, v[c]);
                clear_past(v[c], p.H - (c * NT + t) * 8);
            }
        }
        const float rs = cur.post;
        float s[1] = {0.f};
        if (branch)
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                keep(post[c].w);
                keep(gate[c].w);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float h = cur.b[c].at(i) * rs;
                    s1[c][i] += v[c][i] * h;          // past the end of the row nobody takes it
                    if (p.gate)
                        v[c][i] *= gate[c].at(i);
                    if (p.post)
                        v[c][i] *= post[c].at(i);     // zeros past the end of the row
                    s[0] += v[c][i] * h;
                }
            }
        float m = 0.f;
        if (p.post) {
            row_sum<NT>(s, slots[flip][1]);
            m = s[0] / p.H;
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (c * NT + t) * 8, left = p.H - col;
            keep(cur.b[c].x.w);
            if (left <= 0)
                continue;
            if (p.post)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    v[c][i] = rs * (v[c][i] - cur.b[c].at(i) * rs * m);
            store8(p.db + row * p.lddb + col, left, v[c]);
        }
    }
    if (!p.part)
        return;
    if (RPB > 1) {
        for (int k = 0; k < RPB; ++k) {
            if (sub == k) {
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        // [sum][chunk][i][lane]: consecutive lanes in consecutive banks
                        float *m = meet + ((c * 8 + i) * NT + t);
                        m[0] = k ? m[0] + s2[c][i] : s2[c][i];
                        m[NT * CH * 8] = k ? m[NT * CH * 8] + s1[c][i] : s1[c][i];
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
                s2[c][i] = meet[(c * 8 + i) * NT + t];
                s1[c][i] = meet[(c * 8 + i) * NT + t + NT * CH * 8];
            }
    }
    float *part = p.part + static_cast<int64_t>(blockIdx.x) * 2 * p.H;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (c * NT + t) * 8, left = p.H - col;
        if (left > 0) {
            store8(part + col, left, s2[c]);
            store8(part + p.H + col, left, s1[c]);
        }
    }
}

// Rows past 8192 columns, which with their sums leave no registers: a workgroup
// reads a row for its means and again, from the caches, for the results, and
// adds to its column sums in LDS, or past 16384 columns (LDS_SUMS false) in its
// partial itself; each thread owns its columns.  What bounds it is arithmetic:
// both passes draw the mask and decode.  4096 x 16384 bf16 290 us, of which HBM
// asks 156; with the means in a pass each 1035 x 9984 fp32 took 112, 86 so.
template <typename T, bool JOIN, bool KEPT, bool LDS_SUMS>
__global__ __launch_bounds__(1024, 4) void join_backward_wide_kernel(Bwd<T> p)
{
    extern __shared__ __align__(16) float held[];
    __shared__ float slots[2][3 * 16];
    float *part = p.part ? p.part + static_cast<int64_t>(blockIdx.x) * 2 * p.H : nullptr;
    const int padded = (p.H + 7) / 8 * 8;
    const bool branch = JOIN && (p.post || p.gate);
    // eight columns of sum `which`, added to (first: begun)
    const auto add = [&](int which, int col, int left, bool first, const float (&v)[8]) {
        if (!part)
            return;
        float old[8] = {};
        if constexpr (LDS_SUMS) {
            f32x4 *at = reinterpret_cast<f32x4 *>(held + which * padded + col);
            f32x4 lo = {v[0], v[1], v[2], v[3]}, hi = {v[4], v[5], v[6], v[7]};
            at[0] = first ? lo : at[0] + lo;
            at[1] = first ? hi : at[1] + hi;
        } else {
            if (!first)
                load8(part + which * p.H + col, left, old);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                old[i] += v[i];
            store8(part + which * p.H + col, left, old);
        }
    };
    int flip = 0;
    bool first = true;
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x, flip ^= 1, first = false) {
        const float r2 = p.dy ? p.rstd_pre[row] : 0.f, r1 = JOIN && p.post ? p.rstd_post[row] : 1.f;
        const DropRow d = drop_row(p.drop, row);
        // eight columns of h2 and dy
        const auto after = [&](int col, int left, float (&h)[8], float (&dy)[8]) {
            Src<T, KEPT> x;
            x.load(p.out, p.ldo, p.q_out, row, col, left);
            load8(p.dy + row * p.lddy + col, left, dy);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                h[i] = x.at(i) * r2;
        };
        const auto times = [&](const T *w, int col, int left, float (&v)[8]) {
            float g[8];
            if (!w)
                return;
            load8(w + col, left, g);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                v[i] *= g[i];
        };
        // Both means from one pass: with t0 = dout + rho2 g, t = t0 - rho2 h2 m2,
        // and D and the gains are linear, so the sum of e h1 is that of t0's less
        // rho2 m2 times that of h2's.
        float m2 = 0.f, m1 = 0.f;
        const bool after_mean = p.dy != nullptr, before_mean = JOIN && p.post;
        if (after_mean || before_mean) {
            float s[3] = {0.f, 0.f, 0.f};
#pragma unroll 2
            for (int col = threadIdx.x * 8; col < p.H; col += 8192) {
                const int left = p.H - col;
                float v[8] = {}, h[8] = {}, g[8] = {};
                if (after_mean) {
                    after(col, left, h, g);
                    times(p.pre, col, left, g);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    s[0] += g[i] * h[i];     // past the end of the row g = 0
                if (!before_mean)
                    continue;
                load8(p.dout + row * p.lddo + col, p.dout ? left : 0, v);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    v[i] += r2 * g[i];
                Src<T, KEPT> b;
                b.load(p.b, p.ldb, p.q_b, row, col, left);
                float w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    w[i] = b.at(i) * r1;
                times(p.gate, col, left, w);
                times(p.post, col, left, w);   // zeros past the end of the row
                if (p.drop.below) {
                    drop8(p.drop, d, col, v);
                    clear_past(v, left);
                }
                if (p.drop.below && after_mean) {
                    drop8(p.drop, d, col, h);
                    clear_past(h, left);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    s[1] += v[i] * w[i];
                    s[2] += h[i] * w[i];
                }
            }
            row_sum<1024>(s, slots[flip]);
            m2 = s[0] / p.H;
            // no h2 that counts: of a row that is dropped whole, whose m2 may be NaN
            m1 = (s[2] == 0.f ? s[1] : s[1] - r2 * m2 * s[2]) / p.H;
        }
        // eight columns of t, with dy h2 for the column sums
        const auto whole = [&](int col, int left, float (&v)[8]) {
            load8(p.dout + row * p.lddo + col, p.dout ? left : 0, v);
            if (!p.dy)
                return;
            float h[8], g[8];
            after(col, left, h, g);
            float o[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                o[i] = g[i] * h[i];
            add(0, col, left, first, o);
            times(p.pre, col, left, g);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                v[i] += r2 * (g[i] - h[i] * m2);
        };
        // eight columns of e and h1 from u, with u h1 for the column sums
        const auto before = [&](int col, int left, float (&v)[8], float (&h)[8]) {
            Src<T, KEPT> b;
            b.load(p.b, p.ldb, p.q_b, row, col, left);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                h[i] = b.at(i) * r1;
            float o[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                o[i] = i < left ? v[i] * h[i] : 0.f;
            add(1, col, left, first, o);
            times(p.gate, col, left, v);
            times(p.post, col, left, v);
        };
#pragma unroll 1
        for (int col = threadIdx.x * 8; col < p.H; col += 8192) {
            const int left = p.H - col;
            float v[8], o[8], h[8];
            whole(col, left, v);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                o[i] = JOIN ? p.scale * v[i] : v[i];
            if (JOIN) {
                if (p.drop.below)
                    drop8(p.drop, d, col, v);
                if (branch)
                    before(col, left, v, h);
                if (p.post)
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        v[i] = r1 * (v[i] - h[i] * m1);
            }
            // after everything that is read of these columns: dr and db may take its place
            if (p.dr)
                store8(p.dr + row * p.lddr + col, left, o);
            if (JOIN)
                store8(p.db + row * p.lddb + col, left, v);
        }
    }
    if (!part || (!LDS_SUMS && !first))
        return;
    for (int col = threadIdx.x * 8; col < p.H; col += 8192)
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            // nothing was added where there are no rows, or no such sum
            const bool some = !first && (which ? branch : p.dy != nullptr);
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                v[i] = LDS_SUMS && some ? held[which * padded + col + i] : 0.f;
            store8(part + which * p.H + col, p.H - col, v);
        }
}

// Column sums over the partials, and what the gradients of the gains are of
// them: 64 columns and 16 slices of the partials a workgroup, each slice in
// order, the slices joined in order.
constexpr int kSlices = 16;
struct Gains {
    float *dpre, *dpost, *dgate;
    const void *post, *gate;
    int accumulate;
};
template <typename T>
__global__ __launch_bounds__(64 * kSlices) void join_sums_kernel(const float *part, int n, int H, Gains g)
{
    __shared__ float meet[kSlices][64];
    const int lane = threadIdx.x & 63, sl = threadIdx.x >> 6;
    const int col = blockIdx.x * 64 + lane;       // over 2 H: the columns of dpre, then those of s
    const int per = (n + kSlices - 1) / kSlices, end = min(n, (sl + 1) * per);
    float s = 0.f;
    if (col < 2 * H)
#pragma unroll 8
        for (int i = sl * per; i < end; ++i)
            s += part[static_cast<int64_t>(i) * 2 * H + col];
    meet[sl][lane] = s;
    __syncthreads();
    if (sl || col >= 2 * H)
        return;
    s = meet[0][lane];
#pragma unroll
    for (int i = 1; i < kSlices; ++i)
        s += meet[i][lane];
    const auto put = [&](float *out, int at, float v) {
        if (out)
            out[at] = g.accumulate ? out[at] + v : v;
    };
    const auto gain = [&](const void *p, int at) {
        if (!p)
            return 1.f;
        const T x = static_cast<const T *>(p)[at];
        if constexpr (sizeof(T) == 2)
            return bf16_to_f32(x);
        else
            return x;
    };
    if (col < H) {
        put(g.dpre, col, s);
    } else {
        put(g.dpost, col - H, s * gain(g.gate, col - H));
        put(g.dgate, col - H, s * gain(g.post, col - H));
    }
}

// Threads and chunks for a row of H columns: forward as the layer norm, which
// holds as much; backward one or two chunks, all that its registers hold.
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
        return {256, 1};
    if (H <= 4096)
        return f32 ? Shape{512, 1} : Shape{256, 2};
    if (H <= 8192)
        return f32 ? Shape{1024, 1} : Shape{512, 2};
    return {0, 0};   // the kernel for wide rows
}

// Workgroups of the backward pass, which is also its number of partials: what
// the card holds at once.
inline int bwd_groups(int64_t rows, int H, bool f32)
{
    const int64_t blocks = H <= 1024 ? (rows + 3) / 4 : rows;
    // registers: 105 to 146 a lane for one chunk, to 242 for two
    const int most = H <= 512 ? 1024 : H <= 1024 ? 512 : H <= 2048 ? (f32 ? 768 : 1024) : H <= 4096 && !f32 ? 512 : 256;
    return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(blocks, most)));
}

inline int check_common(int64_t rows, int H, int dt)
{
    ACSC_CHECK_ARG(dt == ACSC_F32 || dt == ACSC_BF16, ACSC_EDTYPE, "unknown dtype %d", dt);
    ACSC_CHECK_ARG(rows >= 0 && rows < (1ll << 31), ACSC_EINVAL, "rows=%lld outside [0, 2^31)", (long long)rows);
    ACSC_CHECK_ARG(H >= 1 && H <= kMaxH, ACSC_EINVAL, "H=%d outside [1, %d]", H, kMaxH);
    return ACSC_OK;
}

// A [rows, H] tensor as a call takes it.
struct Mat {
    const void *p;
    int64_t ld;
    const char *name;
};

inline int check_mat(const Mat &m, int64_t rows, int H, int dt)
{
    ACSC_CHECK_ARG(rows == 0 || m.p, ACSC_EINVAL, "null pointer %s", m.name);
    ACSC_CHECK_ARG(m.ld >= H, ACSC_EINVAL, "ld of %s is %lld < H=%d", m.name, (long long)m.ld, H);
    ACSC_CHECK_ARG(aligned(m.p, dtype_size(static_cast<acsc_dtype>(dt))), ACSC_EALIGN, "%s not aligned to its elements", m.name);
    return ACSC_OK;
}

// An output in the place of an input has its row stride.
inline int check_place(const Mat &o, const Mat &i, int64_t rows)
{
    ACSC_CHECK_ARG(rows == 0 || !o.p || o.p != i.p || o.ld == i.ld, ACSC_EINVAL, "%s in place of %s needs its row stride", o.name, i.name);
    return ACSC_OK;
}

inline int check_gains(const void *p, int dt, const char *name)
{
    ACSC_CHECK_ARG(aligned(p, dtype_size(static_cast<acsc_dtype>(dt))), ACSC_EALIGN, "%s not aligned to its elements", name);
    return ACSC_OK;
}

inline int check_f32(const float *p, const char *name)
{
    ACSC_CHECK_ARG(aligned(p, 4), ACSC_EALIGN, "%s not 4-byte aligned", name);
    return ACSC_OK;
}

#define ACSC_TRY(call)       \
    if (int rc_ = (call))  \
    return rc_

template <typename T, bool JOIN, bool AGAIN>
int run_forward(const Fwd<T> &p, hipStream_t st, const char *tag)
{
    const Shape s = forward_shape(p.H, sizeof(T) == 4);
    const int64_t blocks = s.nt == 64 ? (p.rows + 3) / 4 : p.rows;
    // a grid has under 2^32 threads along x: past 2^20 workgroups it goes on along y
    const int64_t across = std::min<int64_t>(blocks, 1 << 20);
    const dim3 grid(static_cast<unsigned>(across), static_cast<unsigned>((blocks + across - 1) / across));
#define ACSC_CASE(NT, CH)           \
    if (s.nt == NT && s.ch == CH) \
        ACSC_LAUNCH(tag, (join_forward_kernel<T, NT, CH, JOIN, AGAIN>), grid, dim3(NT < 256 ? 256 : NT), 0, st, p);
    ACSC_CASE(64, 1)
    ACSC_CASE(64, 2)
    ACSC_CASE(256, 1)
    ACSC_CASE(1024, 2)
    ACSC_CASE(1024, 4)
    if constexpr (sizeof(T) == 4) {
        ACSC_CASE(512, 1)
        ACSC_CASE(1024, 1)
    } else {
        ACSC_CASE(256, 2)
        ACSC_CASE(512, 2)
    }
#undef ACSC_CASE
    return check_launch(tag);
}

template <typename T, bool JOIN, bool KEPT>
int run_backward(const Bwd<T> &p, int groups, hipStream_t st, const char *tag)
{
    const Shape s = backward_shape(p.H, sizeof(T) == 4);
    const dim3 grid(groups);
#define ACSC_CASE(NT, CH, AHEAD)    \
    if (s.nt == NT && s.ch == CH) \
        ACSC_LAUNCH(tag, (join_backward_kernel<T, NT, CH, JOIN, KEPT, AHEAD>), grid, dim3(NT < 256 ? 256 : NT), 0, st, p);
    ACSC_CASE(64, 1, true)
    ACSC_CASE(64, 2, true)
    ACSC_CASE(256, 1, true)
    if constexpr (sizeof(T) == 4) {
        ACSC_CASE(512, 1, true)
        ACSC_CASE(1024, 1, false)
    } else {
        ACSC_CASE(256, 2, true)
        ACSC_CASE(512, 2, true)
    }
#undef ACSC_CASE
    if (!s.nt) {
        if (p.H <= 16384) {
            const size_t lds = static_cast<size_t>((p.H + 7) / 8 * 8) * 2 * sizeof(float);
            // once a device: asked for on every call it costs the host more than the launch
            static std::atomic<uint64_t> allowed{0};
            int dev = 0;
            if (hipGetDevice(&dev) != hipSuccess)
                return set_error(ACSC_EHIP, "cannot query the device");
            if (dev > 63 || !(allowed.load(std::memory_order_relaxed) >> dev & 1)) {
                if (int rc = allow_lds(join_backward_wide_kernel<T, JOIN, KEPT, true>, 16384 * 2 * sizeof(float)))
                    return rc;
                if (dev < 64)
                    allowed.fetch_or(1ull << dev, std::memory_order_relaxed);
            }
            ACSC_LAUNCH(tag, (join_backward_wide_kernel<T, JOIN, KEPT, true>), grid, dim3(1024), lds, st, p);
        } else {
            ACSC_LAUNCH(tag, (join_backward_wide_kernel<T, JOIN, KEPT, false>), grid, dim3(1024), 0, st, p);
        }
    }
    return check_launch(tag);
}

template <typename T>
const T *as(const void *p)
{
    return static_cast<const T *>(p);
}
template <typename T>
T *as(void *p)
{
    return static_cast<T *>(p);
}

// What join_backward and rms_backward are given, checked.
struct BwdArgs {
    Mat dout, dy, out, b, dr, db;
    const q8_tensor *q_out, *q_b;
    const void *post, *gate, *pre;
    const float *rstd_post, *rstd_pre;
    float *dpost, *dgate, *dpre;
    float scale;
    Drop drop;
    int accumulate;
};

template <typename T>
int launch_backward(const BwdArgs &a, int64_t rows, int H, int groups, float *part, hipStream_t st, const char *tag)
{
    const Bwd<T> p{as<T>(a.dout.p), a.dout.ld, as<T>(a.dy.p), a.dy.ld, as<T>(a.out.p), a.out.ld, q8_of(a.q_out), as<T>(a.b.p), a.b.ld,
                   q8_of(a.q_b), as<T>(a.post), as<T>(a.gate), as<T>(a.pre), a.rstd_post, a.rstd_pre,
                   as<T>(const_cast<void *>(a.dr.p)), a.dr.ld, as<T>(const_cast<void *>(a.db.p)), a.db.ld, part, a.drop, rows, H, a.scale};
    const bool kept = a.q_out || a.q_b;
    int rc;
    if (a.db.p)
        rc = kept ? run_backward<T, true, true>(p, groups, st, tag) : run_backward<T, true, false>(p, groups, st, tag);
    else
        rc = kept ? run_backward<T, false, true>(p, groups, st, tag) : run_backward<T, false, false>(p, groups, st, tag);
    if (rc || !part)
        return rc;
    ACSC_LAUNCH("join_sums", join_sums_kernel<T>, dim3((2 * H + 63) / 64), dim3(64 * kSlices), 0, st, part, groups, H,
                Gains{a.dpre, a.dpost, a.dgate, a.post, a.gate, a.accumulate});
    return check_launch("join_sums");
}

int backward(const BwdArgs &a, acsc_dtype dt, int64_t rows, int H, void *ws, size_t ws_bytes, hipStream_t st, const char *tag)
{
    const bool sums = a.dpost || a.dgate || a.dpre;
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
    return dt == ACSC_BF16 ? launch_backward<uint16_t>(a, rows, H, groups, part, st, tag)
                           : launch_backward<float>(a, rows, H, groups, part, st, tag);
}

}  // namespace
}  // namespace acsc

using namespace acsc;

extern "C" int rms_forward(const void *x, acsc_dtype dt, int64_t rows, int H, int64_t ld_x, const void *gamma, float eps, void *y,
                           int64_t ld_y, float *rstd, const q8_tensor *q, hipStream_t stream)
{
    clear_error();
    ACSC_TRY(check_common(rows, H, dt));
    ACSC_CHECK_ARG(std::isfinite(eps) && eps > 0.f, ACSC_EINVAL, "eps=%g must be positive", eps);
    const Mat mx{x, ld_x, "x"}, my{y, ld_y, "y"};
    ACSC_TRY(check_mat(mx, rows, H, dt));
    ACSC_TRY(check_mat(my, rows, H, dt));
    ACSC_TRY(check_place(my, mx, rows));
    ACSC_TRY(check_gains(gamma, dt, "gamma"));
    ACSC_TRY(check_f32(rstd, "rstd"));
    if (q)
        ACSC_TRY(check_q8(q, rows, H));
    if (rows == 0)
        return ACSC_OK;
    const auto go = [&](auto type) {
        typedef decltype(type) T;
        Fwd<T> p{};
        p.r = as<T>(x);
        p.ldr = ld_x;
        p.pre = as<T>(gamma);
        p.y = as<T>(y);
        p.ldy = ld_y;
        p.rstd_pre = rstd;
        p.q_out = q8_of(q);
        p.rows = rows;
        p.H = H;
        p.eps = eps;
        return run_forward<T, false, false>(p, stream, "rms_forward");
    };
    return dt == ACSC_BF16 ? go(uint16_t{}) : go(float{});
}

extern "C" int rms_recompute(const void *x, int64_t ld_x, const q8_tensor *q, acsc_dtype dt, int64_t rows, int H,
                             const float *rstd, const void *gamma, void *y, int64_t ld_y, hipStream_t stream)
{
    clear_error();
    ACSC_TRY(check_common(rows, H, dt));
    ACSC_CHECK_ARG(rows == 0 || (x != nullptr) != (q != nullptr), ACSC_EINVAL, "exactly one of x and its checkpoint is needed");
    const Mat mx{x, ld_x, "x"}, my{y, ld_y, "y"};
    if (x)
        ACSC_TRY(check_mat(mx, rows, H, dt));
    if (q)
        ACSC_TRY(check_q8(q, rows, H));
    ACSC_TRY(check_mat(my, rows, H, dt));
    ACSC_TRY(check_place(my, mx, rows));
    ACSC_CHECK_ARG(rows == 0 || rstd, ACSC_EINVAL, "null pointer rstd");
    ACSC_TRY(check_f32(rstd, "rstd"));
    ACSC_TRY(check_gains(gamma, dt, "gamma"));
    if (rows == 0)
        return ACSC_OK;
    const auto go = [&](auto type) {
        typedef decltype(type) T;
        Fwd<T> p{};
        p.r = as<T>(x);
        p.ldr = ld_x;
        p.src = q8_of(q);
        p.pre = as<T>(gamma);
        p.y = as<T>(y);
        p.ldy = ld_y;
        p.rstd_pre = const_cast<float *>(rstd);   // read only there
        p.rows = rows;
        p.H = H;
        return run_forward<T, false, true>(p, stream, "rms_recompute");
    };
    return dt == ACSC_BF16 ? go(uint16_t{}) : go(float{});
}

extern "C" int join_workspace_size(int64_t rows, int H, size_t *bytes)
{
    clear_error();
    ACSC_TRY(check_common(rows, H, ACSC_F32));
    ACSC_CHECK_ARG(bytes, ACSC_EINVAL, "null pointer bytes");
    *bytes = static_cast<size_t>(std::max(bwd_groups(rows, H, false), bwd_groups(rows, H, true))) * 2 * H * sizeof(float);
    return ACSC_OK;
}

extern "C" int rms_backward(const void *dy, int64_t ld_dy, const void *x, int64_t ld_x, const q8_tensor *q, acsc_dtype dt,
                            int64_t rows, int H, const float *rstd, const void *gamma, const void *add, int64_t ld_add,
                            void *dx, int64_t ld_dx, float *dgamma, int accumulate, void *ws, size_t ws_bytes,
                            hipStream_t stream)
{
    clear_error();
    ACSC_TRY(check_common(rows, H, dt));
    ACSC_CHECK_ARG(rows == 0 || (x != nullptr) != (q != nullptr), ACSC_EINVAL, "exactly one of x and its checkpoint is needed");
    BwdArgs a{};
    a.dy = {dy, ld_dy, "dy"};
    a.out = {x, ld_x, "x"};
    a.q_out = q;
    a.dout = {add, ld_add, "add"};
    a.dr = {dx, ld_dx, "dx"};
    a.pre = gamma;
    a.rstd_pre = rstd;
    a.dpre = dgamma;
    a.accumulate = accumulate;
    ACSC_TRY(check_mat(a.dy, rows, H, dt));
    if (x)
        ACSC_TRY(check_mat(a.out, rows, H, dt));
    if (q)
        ACSC_TRY(check_q8(q, rows, H));
    if (add)
        ACSC_TRY(check_mat(a.dout, rows, H, dt));
    ACSC_TRY(check_mat(a.dr, rows, H, dt));
    for (const Mat *in : {&a.dy, &a.out, &a.dout})
        ACSC_TRY(check_place(a.dr, *in, rows));
    ACSC_CHECK_ARG(rows == 0 || rstd, ACSC_EINVAL, "null pointer rstd");
    ACSC_TRY(check_f32(rstd, "rstd"));
    ACSC_TRY(check_f32(dgamma, "dgamma"));
    ACSC_TRY(check_gains(gamma, dt, "gamma"));
    return backward(a, dt, rows, H, ws, ws_bytes, stream, "rms_backward");
}

extern "C" int join_forward(const void *r, int64_t ld_r, const void *b, int64_t ld_b, acsc_dtype dt, int64_t rows, int H,
                            const void *post, const void *gate, float scale, const drop_mask *drop, const void *pre, float eps,
                            void *out, int64_t ld_out, void *y, int64_t ld_y, float *rstd_post, float *rstd_pre,
                            const q8_tensor *q_out, const q8_tensor *q_b, hipStream_t stream)
{
    clear_error();
    ACSC_TRY(check_common(rows, H, dt));
    ACSC_CHECK_ARG(std::isfinite(eps) && eps > 0.f, ACSC_EINVAL, "eps=%g must be positive", eps);
    ACSC_CHECK_ARG(std::isfinite(scale), ACSC_EINVAL, "scale=%g must be finite", scale);
    Drop d;
    ACSC_TRY(drop_of(drop, rows, H, &d));
    const Mat mr{r, ld_r, "r"}, mb{b, ld_b, "b"}, mo{out, ld_out, "out"}, my{y, ld_y, "y"};
    for (const Mat *m : {&mr, &mb, &mo})
        ACSC_TRY(check_mat(*m, rows, H, dt));
    if (y)
        ACSC_TRY(check_mat(my, rows, H, dt));
    for (const Mat *in : {&mr, &mb}) {
        ACSC_TRY(check_place(mo, *in, rows));
        ACSC_TRY(check_place(my, *in, rows));
    }
    ACSC_CHECK_ARG(rows == 0 || out != y, ACSC_EINVAL, "out and y must not overlap");
    ACSC_CHECK_ARG(y || rows == 0 || (!pre && !rstd_pre), ACSC_EINVAL, "pre or rstd_pre without y");
    ACSC_CHECK_ARG(post || !rstd_post, ACSC_EINVAL, "rstd_post without post");
    ACSC_TRY(check_gains(post, dt, "post"));
    ACSC_TRY(check_gains(gate, dt, "gate"));
    ACSC_TRY(check_gains(pre, dt, "pre"));
    ACSC_TRY(check_f32(rstd_post, "rstd_post"));
    ACSC_TRY(check_f32(rstd_pre, "rstd_pre"));
    if (q_out)
        ACSC_TRY(check_q8(q_out, rows, H));
    if (q_b)
        ACSC_TRY(check_q8(q_b, rows, H));
    if (rows == 0)
        return ACSC_OK;
    const Q8 none = q8_of(nullptr);
    const auto go = [&](auto type) {
        typedef decltype(type) T;
        return run_forward<T, true, false>({as<T>(r), ld_r, as<T>(b), ld_b, none, as<T>(post), as<T>(gate), as<T>(pre),
                                            as<T>(out), ld_out, as<T>(y), ld_y, rstd_post, rstd_pre, q8_of(q_out), q8_of(q_b), d,
                                            rows, H, scale, eps}, stream, "join_forward");
    };
    return dt == ACSC_BF16 ? go(uint16_t{}) : go(float{});
}

extern "C" int join_backward(const void *dout, int64_t ld_dout, const void *dy, int64_t ld_dy, const void *out, int64_t ld_out,
                             const q8_tensor *q_out, const void *b, int64_t ld_b, const q8_tensor *q_b, acsc_dtype dt,
                             int64_t rows, int H, const void *post, const void *gate, float scale, const drop_mask *drop,
                             const void *pre, const float *rstd_post, const float *rstd_pre, void *dr, int64_t ld_dr, void *db,
                             int64_t ld_db, float *dpost, float *dgate, float *dpre, int accumulate, void *ws, size_t ws_bytes,
                             hipStream_t stream)
{
    clear_error();
    ACSC_TRY(check_common(rows, H, dt));
    ACSC_CHECK_ARG(std::isfinite(scale), ACSC_EINVAL, "scale=%g must be finite", scale);
    BwdArgs a{};
    ACSC_TRY(drop_of(drop, rows, H, &a.drop));
    a.dout = {dout, ld_dout, "dout"};
    a.dy = {dy, ld_dy, "dy"};
    a.out = {out, ld_out, "out"};
    a.b = {b, ld_b, "b"};
    a.dr = {dr, ld_dr, "dr"};
    a.db = {db, ld_db, "db"};
    a.q_out = q_out;
    a.q_b = q_b;
    a.post = post;
    a.gate = gate;
    a.pre = pre;
    a.rstd_post = rstd_post;
    a.rstd_pre = rstd_pre;
    a.dpost = dpost;
    a.dgate = dgate;
    a.dpre = dpre;
    a.scale = scale;
    a.accumulate = accumulate;
    ACSC_CHECK_ARG(rows == 0 || dout || dy, ACSC_EINVAL, "one of dout and dy is needed");
    ACSC_CHECK_ARG(!out || !q_out, ACSC_EINVAL, "out and its checkpoint are both given");
    ACSC_CHECK_ARG(!b || !q_b, ACSC_EINVAL, "b and its checkpoint are both given");
    ACSC_CHECK_ARG(!dy || rows == 0 || out || q_out, ACSC_EINVAL, "dy needs out or its checkpoint");
    ACSC_CHECK_ARG(!dy || rows == 0 || rstd_pre, ACSC_EINVAL, "null pointer rstd_pre");
    ACSC_CHECK_ARG(dy || rows == 0 || !dpre, ACSC_EINVAL, "dpre without dy");
    ACSC_CHECK_ARG((!post && !gate) || rows == 0 || b || q_b, ACSC_EINVAL, "post and gate need b or its checkpoint");
    ACSC_CHECK_ARG(!post || rows == 0 || rstd_post, ACSC_EINVAL, "null pointer rstd_post");
    ACSC_CHECK_ARG(post || !dpost, ACSC_EINVAL, "dpost without post");
    ACSC_CHECK_ARG(gate || !dgate, ACSC_EINVAL, "dgate without gate");
    ACSC_CHECK_ARG(!dy || (!post && !gate) || (!(out && q_b) && !(b && q_out)), ACSC_EINVAL,
                   "out and b must both be tensors or both be checkpoints");
    for (const Mat *m : {&a.dout, &a.dy, &a.out, &a.b, &a.dr})
        if (m->p)
            ACSC_TRY(check_mat(*m, rows, H, dt));
    ACSC_TRY(check_mat(a.db, rows, H, dt));
    if (q_out)
        ACSC_TRY(check_q8(q_out, rows, H));
    if (q_b)
        ACSC_TRY(check_q8(q_b, rows, H));
    for (const Mat *in : {&a.dout, &a.dy, &a.out, &a.b}) {
        ACSC_TRY(check_place(a.dr, *in, rows));
        ACSC_TRY(check_place(a.db, *in, rows));
    }
    ACSC_CHECK_ARG(rows == 0 || dr != db, ACSC_EINVAL, "dr and db must not overlap");
    ACSC_TRY(check_gains(post, dt, "post"));
    ACSC_TRY(check_gains(gate, dt, "gate"));
    ACSC_TRY(check_gains(pre, dt, "pre"));
    for (const float *f : {rstd_post, rstd_pre, static_cast<const float *>(dpost), static_cast<const float *>(dgate),
                           static_cast<const float *>(dpre)})
        ACSC_TRY(check_f32(f, "an fp32 array"));
    // a source that the formula does not read has no say in which kernel runs
    if (!dy)
        a.q_out = nullptr, a.out.p = nullptr;
    if (!post && !gate)
        a.q_b = nullptr, a.b.p = nullptr;
    return backward(a, dt, rows, H, ws, ws_bytes, stream, "join_backward");
}
