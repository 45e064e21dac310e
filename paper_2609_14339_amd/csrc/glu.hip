// The gated linear layer, h = act(x Wg^T + bg) (x Wu^T + bu): the entry points,
// the sum of a cut product's pieces, and the gradient through the gate alone.
//
// With dh the gradient of h, and g and u the pre-activations:
//   dg = dh u act'(g),  du = dh act(g),  dx = (dg, du) (Wg; Wu),  dW = (dg, du)^T x
// so that with dz = (dg, du) in one tensor and the two weights in one, the rest
// of the gradient is a linear layer's.  The bias gradient is summed from dz
// before its rounding, in the epilogue or the pass that forms it (from the
// rounded dz it is 1e-3 off in bf16).
#include "lin_plan.h"

namespace acsc {
namespace {

// Pieces of tiles: a workgroup takes 2048 hidden columns' worth of rows, a
// thread eight columns, of units of UH columns: a tile's 64 or 128, or with a
// checkpoint two tiles of 64, so that sixteen lanes hold a group.
template <typename TO, int TM, int T, int UH>
__global__ __launch_bounds__(256) void glu_join_kernel(Gemm g)
{
    constexpr int TC = T / 2, PER = TM * UH / 2048, SPAN = UH / TC;   // tiles of a unit
    const int64_t count = static_cast<int64_t>(g.tm) * g.tn - g.whole, unit = blockIdx.x / PER;
    const int c = (blockIdx.x % PER) * 256 + threadIdx.x, row = c / (UH / 8);
    int col = c % (UH / 8) * 8, tile_m, tile_n;
    int64_t id = unit;
    if (SPAN > 1) {
        // every tile is cut; the pairs of a row of tiles follow one another
        const int pairs = (g.tn + 1) / 2;
        tile_m = static_cast<int>(unit / pairs);
        tile_n = static_cast<int>(unit % pairs) * 2 + col / TC;
        col %= TC;
        const int band = tile_m / 4, height = min(g.tm - band * 4, 4);
        id = static_cast<int64_t>(band) * 4 * g.tn + static_cast<int64_t>(tile_n) * height + tile_m % 4;
    } else {
        tile_at(g, g.whole + id, tile_m, tile_n);
    }
    const int64_t m = static_cast<int64_t>(tile_m) * TM + row;
    const int n = tile_n * TC + col, left = m < g.M ? g.N - n : 0;
    float vg[8] = {}, vu[8] = {}, bg[8], bu[8];
    if (left > 0) {
        const float *p = g.part + (id * TM + row) * T + col / 64 * 128 + col % 64;
        add_pieces(p, count * TM * T, g.splits, vg);
        add_pieces(p + 64, count * TM * T, g.splits, vu);
    }
    glu_bias<TO>(g.e, g.N, n, bg, bu);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        vg[i] += bg[i];
        vu[i] += bu[i];
    }
    glu_epilogue<TO>(g.e, g.N, vg, vu, GluAt<TO>(g.e, m, n), n, left);
}

// Pieces of a product for few tokens: 2048 columns of a row a workgroup.
template <typename TO>
__global__ __launch_bounds__(256) void glu_join_few_kernel(Gemm g)
{
    const int64_t m = blockIdx.y, step = g.M * 2 * g.ldp;
    const int n = (blockIdx.x * 256 + threadIdx.x) * 8, left = g.N - n;
    float vg[8] = {}, vu[8] = {}, bg[8], bu[8];
    if (left > 0) {
        const float *p = g.part + m * 2 * g.ldp + n;
        add_pieces(p, step, g.splits, vg);
        add_pieces(p + g.ldp, step, g.splits, vu);
    }
    glu_bias<TO>(g.e, g.N, n, bg, bu);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        vg[i] += bg[i];
        vu[i] += bu[i];
    }
    glu_epilogue<TO>(g.e, g.N, vg, vu, GluAt<TO>(g.e, m, n), n, left);
}

// Pieces of dh, then the gate's gradient.
template <typename TO, int TM, int T>
__global__ __launch_bounds__(256) void glu_gate_join_kernel(Gemm g)
{
    constexpr int PER = TM * T / 2048, ROWS = 2048 / T;
    __shared__ float meet[ROWS][2][T];
    const int64_t id = blockIdx.x / PER, count = static_cast<int64_t>(g.tm) * g.tn - g.whole;
    const int c = (blockIdx.x % PER) * 256 + threadIdx.x, row = c / (T / 8), col = c % (T / 8) * 8;
    int tile_m, tile_n;
    tile_at(g, g.whole + id, tile_m, tile_n);
    const int64_t m = static_cast<int64_t>(tile_m) * TM + row;
    const int n = tile_n * T + col, left = m < g.M ? g.N - n : 0;
    float sg[8] = {}, su[8] = {};
    if (left > 0) {
        float v[8];
        add_pieces(g.part + (id * TM + row) * T + col, count * TM * T, g.splits, v);
        GluBeside<TO> beside;
        const GluAt<TO> at(g.e, m, n);
        load_glu_beside<TO>(g.e, g.N, beside, at, left);
        glu_gate_epilogue<TO>(g.e, g.N, v, beside, at, left, sg, su);
    }
    if (!g.e.sums)
        return;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        meet[row % ROWS][0][col + i] = sg[i];
        meet[row % ROWS][1][col + i] = su[i];
    }
    __syncthreads();
    float *out = g.e.sums + (g.tm + static_cast<int64_t>(tile_m - g.e.cut_first) * g.e.cut_slots + blockIdx.x % PER) * 2 * g.N;
    for (int k = threadIdx.x; k < 2 * T; k += 256) {
        float s = 0.f;
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
            s += meet[r][k / T][k % T];
        if (tile_n * T + k % T < g.N)
            out[static_cast<int64_t>(k / T) * g.N + tile_n * T + k % T] = s;
    }
}

// The column sums' partials, in order: 64 columns and 16 slices of the rows of
// tiles a workgroup, the slices joined in order.
constexpr int kSlices = 16;
__global__ __launch_bounds__(64 * kSlices) void glu_sums_kernel(Gemm g, int tile, float *db, int accumulate)
{
    __shared__ float meet[kSlices][64];
    const int lane = threadIdx.x & 63, sl = threadIdx.x >> 6, F = g.N;
    const int col = blockIdx.x * 64 + lane, n = col % F;      // over 2 F
    const int per = (g.tm + kSlices - 1) / kSlices, end = min(g.tm, (sl + 1) * per);
    float s = 0.f;
    if (col < 2 * F)
        for (int m = sl * per; m < end; ++m) {
            const int band = m / 4, height = min(g.tm - band * 4, 4);
            const int64_t id = static_cast<int64_t>(band) * 4 * g.tn + static_cast<int64_t>(n / tile) * height + m % 4;
            const bool whole = id < g.whole;
            const int slots = whole ? 1 : g.e.cut_slots;
            const int64_t at = whole ? m : g.tm + static_cast<int64_t>(m - g.e.cut_first) * slots;
            const float *p = g.e.sums + at * 2 * F + col;
            for (int i = 0; i < slots; ++i)
                s += p[static_cast<int64_t>(i) * 2 * F];
        }
    meet[sl][lane] = s;
    __syncthreads();
    if (sl || col >= 2 * F)
        return;
    s = meet[0][lane];
#pragma unroll
    for (int i = 1; i < kSlices; ++i)
        s += meet[i][lane];
    db[col] = accumulate ? db[col] + s : s;
}

__global__ __launch_bounds__(256) void glu_zero_kernel(float *y, int n)
{
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < n)
        y[i] = 0.f;
}

// The gate's gradient of a given dh: a wave takes 512 columns of a row, eight a
// lane.
template <typename T>
__global__ __launch_bounds__(256) void glu_act_kernel(const T *dh, int64_t lddh, int64_t rows, int F, Epi e)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int segs = (F + 511) / 512;
    for (int64_t w = static_cast<int64_t>(blockIdx.x) * 4 + wave; w < rows * segs; w += static_cast<int64_t>(gridDim.x) * 4) {
        const int64_t row = w / segs;
        const int col = static_cast<int>(w - row * segs) * 512 + lane * 8, left = F - col;
        if (left <= 0)
            continue;
        float v[8];
        load8(dh + row * lddh + col, left, v);
        GluBeside<T> beside;
        const GluAt<T> at(e, row, col);
        load_glu_beside<T>(e, F, beside, at, left);
        float sg[8] = {}, su[8] = {};
        glu_gate_epilogue<T>(e, F, v, beside, at, left, sg, su);
    }
}

// The same with the column sums of both halves before their rounding: a
// workgroup takes 512 columns of `per` rows, every fourth row a wave; its waves
// meet in LDS in order and it leaves one partial, [2][F], or the result where
// there is one workgroup along the rows.  HBM bounds it: 8192 x 14336 bf16, z
// kept, 250 us with the partials' sum, 4.7 TB/s (205 without sums, partly from
// the caches, and 68 for those of the rounded dz in a pass of their own).
template <typename T>
__global__ __launch_bounds__(256) void glu_act_sums_kernel(const T *dh, int64_t lddh, int64_t rows, int F, Epi e, int64_t per,
                                                           int accumulate)
{
    __shared__ float meet[4][2][512];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int col = blockIdx.x * 512 + lane * 8, left = F - col;
    const int64_t end = min(rows, (blockIdx.y + static_cast<int64_t>(1)) * per);
    float sg[8] = {}, su[8] = {};
    if (left > 0)
        for (int64_t row = blockIdx.y * per + wave; row < end; row += 4) {
            float v[8];
            load8(dh + row * lddh + col, left, v);
            GluBeside<T> beside;
            const GluAt<T> at(e, row, col);
            load_glu_beside<T>(e, F, beside, at, left);
            glu_gate_epilogue<T>(e, F, v, beside, at, left, sg, su);
        }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        // consecutive lanes in consecutive banks
        meet[wave][0][i * 64 + lane] = sg[i];
        meet[wave][1][i * 64 + lane] = su[i];
    }
    __syncthreads();
    float *out = e.sums + blockIdx.y * static_cast<int64_t>(2) * F;
    for (int c = threadIdx.x; c < 1024; c += 256) {
        const int half = c / 512, k = c % 512, at = (k & 7) * 64 + (k >> 3), n = blockIdx.x * 512 + k;
        if (n < F) {
            const float s = ((meet[0][half][at] + meet[1][half][at]) + meet[2][half][at]) + meet[3][half][at];
            float *to = out + static_cast<int64_t>(half) * F + n;
            *to = accumulate ? *to + s : s;
        }
    }
}

// Partials of those sums: about eight workgroups a CU, of 16 rows at least; and their bytes.
inline int act_partials(int64_t rows, int F)
{
    const int segs = (F + 511) / 512;
    return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>((rows + 15) / 16, 2048 / segs)));
}
inline size_t act_bytes(int64_t rows, int F)
{
    const int parts = act_partials(rows, F);
    return parts > 1 ? up256(static_cast<size_t>(parts) * 2 * F * sizeof(float)) : 0;
}

template <typename TO, int TM, int T>
void launch_join(const Gemm &g, EpiKind kind, hipStream_t st)
{
    const int64_t tail = static_cast<int64_t>(g.tm) * g.tn - g.whole;
    if (kind == kGluGate) {
        ACSC_LAUNCH("glu_join", (glu_gate_join_kernel<TO, TM, T>), dim3(static_cast<unsigned>(tail * (TM * T / 2048))), dim3(256), 0,
                    st, g);
        return;
    }
    if constexpr (T >= 128) {
        if (T == 128 && g.e.q.codes) {
            const int64_t units = static_cast<int64_t>(g.tm) * ((g.tn + 1) / 2);
            ACSC_LAUNCH("glu_join", (glu_join_kernel<TO, TM, T, 128>), dim3(static_cast<unsigned>(units * (TM * 128 / 2048))),
                        dim3(256), 0, st, g);
        } else {
            ACSC_LAUNCH("glu_join", (glu_join_kernel<TO, TM, T, T / 2>), dim3(static_cast<unsigned>(tail * (TM * (T / 2) / 2048))),
                        dim3(256), 0, st, g);
        }
    }
}

template <typename TO>
void join_tiles(const Gemm &g, const Plan &p, EpiKind kind, hipStream_t st)
{
    if (p.rows == 256)
        launch_join<TO, 256, 256>(g, kind, st);
    else if (p.tile == 64)
        launch_join<TO, 128, 64>(g, kind, st);
    else if (p.rows == 128)
        launch_join<TO, 128, 128>(g, kind, st);
    else if (p.rows == 64)
        launch_join<TO, 64, 128>(g, kind, st);
    else
        launch_join<TO, 32, 128>(g, kind, st);
}

// Host checks of kept pre-activations: z [rows, 2 F] or both checkpoints.
inline int check_kept_pair(const void *z, int64_t ld_z, const q8_tensor *qg, const q8_tensor *qu, int64_t rows, int F, int dt)
{
    ACSC_CHECK_ARG(rows == 0 || (z != nullptr) != (qg != nullptr && qu != nullptr), ACSC_EINVAL,
                   "exactly one of z and the pair of its checkpoints is needed");
    ACSC_CHECK_ARG((qg != nullptr) == (qu != nullptr), ACSC_EINVAL, "one checkpoint of the pair is missing");
    if (z)
        return check_mat(z, true, ld_z, 2 * F, dt, "z");
    if (!qg)
        return ACSC_OK;
    if (int rc = check_q8(qg, rows, F))
        return rc;
    return check_q8(qu, rows, F);
}

inline int check_glu(int64_t rows, int n_in, int F, int dt)
{
    if (int rc = check_layer(rows, n_in, F, dt))
        return rc;
    ACSC_CHECK_ARG(F <= (1 << 21), ACSC_EINVAL, "F=%d outside [1, 2^21]", F);
    return ACSC_OK;
}

// The largest launches: of tiles, and with a checkpoint of the sum of pieces
// that every narrow tile goes through.
inline int check_launches(const Plan &p, bool codes)
{
    if (int rc = check_tiles(p))
        return rc;
    const int64_t groups = static_cast<int64_t>(p.tm) * ((p.tn + 1) / 2) * (p.rows * 128 / 2048);
    ACSC_CHECK_ARG(p.few || !codes || p.tile != 128 || groups * 256 < (1ll << 32), ACSC_EINVAL,
                   "product too large: %lld workgroups for its checkpoint", (long long)groups);
    return ACSC_OK;
}

// The plan of a product, with the operands' copies that bits 0 (A) and 1 (B) of
// `copies` add to those that are needed whatever the alignment.
int plan_glu(glu_op op, int64_t rows, int n_in, int F, acsc_dtype dt, bool codes, int copies, Plan &p)
{
    const EpiKind kind = op == GLU_FORWARD ? kGluForward : kGluGate;
    // the gradient's product is the down projection's: its inputs are the F hidden columns
    const Shape s = op == GLU_FORWARD ? shape_of(kind, rows, n_in, F) : shape_of(kind, rows, F, n_in);
    const auto best = [&](bool col, int64_t inner) {
        return readable(Operand{nullptr, dt == ACSC_F32 ? inner : (inner + 1) / 2 * 2}, col, inner, dt);
    };
    const bool a = best(s.acol, s.acol ? s.M : s.K), b = best(s.bcol, s.bcol ? s.N : s.K);
    p = plan_of(kind, s, dt, a && !(copies & 1), b && !(copies & 2), codes);
    return check_launches(p, codes);
}

// Partials of the column sums: of a cut tile, one for each workgroup of its
// pieces' sum.
inline int cut_slots(const Plan &p) { return p.rows * p.tile / 2048; }
inline int cut_first(const Plan &p)
{
    return p.whole < static_cast<int64_t>(p.tm) * p.tn ? static_cast<int>(p.whole / (4ll * p.tn) * 4) : p.tm;
}
inline size_t sums_bytes(const Plan &p, int F)
{
    const size_t partials = p.tm + static_cast<size_t>(p.tm - cut_first(p)) * cut_slots(p);
    return up256(partials * 2 * F * sizeof(float));
}

int workspace_size(glu_op op, int64_t rows, int n_in, int F, acsc_dtype dt, int extra, bool any, size_t *bytes)
{
    clear_error();
    if (int rc = check_glu(rows, n_in, F, dt))
        return rc;
    ACSC_CHECK_ARG(bytes, ACSC_EINVAL, "null pointer to the result");
    ACSC_CHECK_ARG(op == GLU_FORWARD || op == GLU_BACKWARD_INPUT, ACSC_EINVAL, "unknown product %d", (int)op);
    *bytes = 0;
    if (rows == 0)
        return ACSC_OK;
    // with any alignment: the most that either operand's copy, or its absence, takes
    size_t most = 0;
    for (int copies = 0; copies < (any ? 4 : 1); ++copies) {
        Plan p;
        if (int rc = plan_glu(op, rows, n_in, F, dt, op == GLU_FORWARD && extra, copies, p))
            return rc;
        most = std::max(most, p.bytes() + (op == GLU_BACKWARD_INPUT && extra ? sums_bytes(p, F) : 0));
    }
    *bytes = most;
    return ACSC_OK;
}

// What the gradient of a given dh is asked for: its checks, and the epilogue's arguments.
inline int check_backward_act(const void *dh, int64_t ld_dh, const void *z, int64_t ld_z, const q8_tensor *q_gate,
                              const q8_tensor *q_up, acsc_dtype dt, int64_t rows, int F, acsc_act act, const void *dz, int64_t ld_dz,
                              const void *h, int64_t ld_h)
{
    if (int rc = check_glu(rows, 1, F, dt))
        return rc;
    if (int rc = check_act(act))
        return rc;
    const bool some = rows > 0;
    if (int rc = check_mat(dh, some, ld_dh, F, dt, "dh"))
        return rc;
    if (int rc = check_kept_pair(z, ld_z, q_gate, q_up, rows, F, dt))
        return rc;
    if (int rc = check_mat(dz, some, ld_dz, 2 * F, dt, "dz"))
        return rc;
    if (h)
        if (int rc = check_mat(h, some, ld_h, F, dt, "h"))
            return rc;
    ACSC_CHECK_ARG(!some || (dz != dh && dz != h), ACSC_EINVAL, "dz must not overlap dh or h");
    ACSC_CHECK_ARG(!some || dz != z || ld_dz == ld_z, ACSC_EINVAL, "dz in place of z needs ld_dz == ld_z");
    ACSC_CHECK_ARG(!some || !h || h != dh || ld_h == ld_dh, ACSC_EINVAL, "h in place of dh needs ld_h == ld_dh");
    ACSC_CHECK_ARG(!some || !h || h != z, ACSC_EINVAL, "h must not overlap z");
    return ACSC_OK;
}
inline Epi epi_backward_act(const void *z, int64_t ld_z, const q8_tensor *q_gate, const q8_tensor *q_up, acsc_act act, void *dz,
                            int64_t ld_dz, void *h, int64_t ld_h)
{
    Epi e{};
    e.y = dz;
    e.ldy = ld_dz;
    e.z = const_cast<void *>(z);
    e.ldz = ld_z;
    e.q = q8_of(q_gate);
    e.q_up = q8_of(q_up);
    e.act = act;
    e.hidden = h;
    e.ldh = ld_h;
    return e;
}

}  // namespace

void glu_join_run(const Gemm &g, const Plan &p, EpiKind kind, acsc_dtype dt, hipStream_t st)
{
    const bool b = dt == ACSC_BF16;
    if (p.few) {
        const dim3 grid((g.N + 2047) / 2048, static_cast<unsigned>(g.M));
        if (b)
            ACSC_LAUNCH("glu_join", glu_join_few_kernel<uint16_t>, grid, dim3(256), 0, st, g);
        else
            ACSC_LAUNCH("glu_join", glu_join_few_kernel<float>, grid, dim3(256), 0, st, g);
    } else if (b) {
        join_tiles<uint16_t>(g, p, kind, st);
    } else {
        join_tiles<float>(g, p, kind, st);
    }
}

}  // namespace acsc

using namespace acsc;

extern "C" int glu_workspace_size(glu_op op, int64_t rows, int n_in, int F, acsc_dtype dt, int extra, size_t *bytes)
{
    return workspace_size(op, rows, n_in, F, dt, extra, false, bytes);
}

extern "C" int glu_workspace_size_unaligned(glu_op op, int64_t rows, int n_in, int F, acsc_dtype dt, int extra, size_t *bytes)
{
    return workspace_size(op, rows, n_in, F, dt, extra, true, bytes);
}

extern "C" int glu_product_plan(glu_op op, int64_t rows, int n_in, int F, acsc_dtype dt, int extra, lin_plan *plan)
{
    clear_error();
    if (int rc = check_glu(rows, n_in, F, dt))
        return rc;
    ACSC_CHECK_ARG(plan, ACSC_EINVAL, "null pointer to the result");
    ACSC_CHECK_ARG(op == GLU_FORWARD || op == GLU_BACKWARD_INPUT, ACSC_EINVAL, "unknown product %d", (int)op);
    *plan = lin_plan{};
    if (rows == 0)
        return ACSC_OK;
    Plan p;
    if (int rc = plan_glu(op, rows, n_in, F, dt, op == GLU_FORWARD && extra, 0, p))
        return rc;
    *plan = {p.rows, p.tile, p.whole, static_cast<int64_t>(p.tm) * p.tn - p.whole, p.splits};
    return ACSC_OK;
}

extern "C" int glu_forward(const void *x, int64_t ld_x, acsc_dtype dt, int64_t rows, int n_in, int F, const void *W, int64_t ld_w,
                           const void *bias, acsc_act act, void *h, int64_t ld_h, void *z, int64_t ld_z, const q8_tensor *q_gate,
                           const q8_tensor *q_up, void *ws, size_t ws_bytes, hipStream_t stream)
{
    clear_error();
    if (int rc = check_glu(rows, n_in, F, dt))
        return rc;
    if (int rc = check_act(act))
        return rc;
    const bool some = rows > 0;
    if (int rc = check_mat(x, some, ld_x, n_in, dt, "x"))
        return rc;
    if (int rc = check_mat(W, some, ld_w, n_in, dt, "W"))
        return rc;
    if (int rc = check_mat(h, some, ld_h, F, dt, "h"))
        return rc;
    ACSC_CHECK_ARG(aligned(bias, dtype_size(dt)), ACSC_EALIGN, "bias not aligned to its elements");
    if (z)
        if (int rc = check_mat(z, some, ld_z, 2 * F, dt, "z"))
            return rc;
    ACSC_CHECK_ARG(!some || (h != x && h != W && h != z), ACSC_EINVAL, "h must not overlap x, W or z");
    ACSC_CHECK_ARG(!some || !z || (z != x && z != W), ACSC_EINVAL, "z must not overlap x or W");
    ACSC_CHECK_ARG((q_gate != nullptr) == (q_up != nullptr), ACSC_EINVAL, "one checkpoint of the pair is missing");
    for (const q8_tensor *q : {q_gate, q_up})
        if (q)
            if (int rc = check_q8(q, rows, F))
                return rc;
    if (!some)
        return ACSC_OK;
    Operand w{W, ld_w};
    Shape s = shape_of(kGluForward, rows, n_in, F);
    Plan p = plan_of(kGluForward, s, dt, readable({x, ld_x}, false, n_in, dt), readable(w, false, n_in, dt), q_gate != nullptr);
    if (int rc = check_launches(p, q_gate != nullptr))
        return rc;
    if (int rc = check_ws(ws, ws_bytes, p.bytes()))
        return rc;
    const int64_t es = static_cast<int64_t>(dtype_size(dt));
    // rows of the tensors from `row` on
    const auto product = [&](int64_t row) {
        const auto from = [&](const void *t, int64_t ld) { return t ? static_cast<const char *>(t) + row * ld * es : nullptr; };
        const auto out = [&](void *t, int64_t ld) { return t ? static_cast<char *>(t) + row * ld * es : nullptr; };
        const auto codes = [&](const q8_tensor *q) {
            return q ? Q8{q->codes + row * q->ld_codes, q->scales + row * q->ld_scales, q->ld_codes, q->ld_scales} : q8_of(q);
        };
        Gemm g{};
        g.A = {from(x, ld_x), ld_x};
        g.B = w;
        g.e = Epi{out(h, ld_h), ld_h, bias, nullptr, 0, out(z, ld_z), ld_z, codes(q_gate), act, 0, codes(q_up), nullptr, 0, nullptr, 0, 0};
        const int rc = run_product(g, kGluForward, p, s, dt, dt, static_cast<char *>(ws), nullptr, nullptr, stream, "glu_forward");
        w = g.B;   // where it was copied, the next run finds the copy
        p.pack_b = false;
        return rc;
    };
    if (p.band == p.tm)
        return product(0);
    // runs that take the workspace in turn
    for (int first = 0, tm = p.tm; first < tm; first += p.band) {
        const int64_t row = static_cast<int64_t>(first) * p.rows;
        p.tm = std::min(p.band, tm - first);
        s.M = std::min(static_cast<int64_t>(p.tm) * p.rows, rows - row);
        if (int rc = product(row))
            return rc;
    }
    return ACSC_OK;
}

extern "C" int glu_backward_act(const void *dh, int64_t ld_dh, const void *z, int64_t ld_z, const q8_tensor *q_gate,
                                const q8_tensor *q_up, acsc_dtype dt, int64_t rows, int F, acsc_act act, void *dz, int64_t ld_dz,
                                void *h, int64_t ld_h, hipStream_t stream)
{
    clear_error();
    if (int rc = check_backward_act(dh, ld_dh, z, ld_z, q_gate, q_up, dt, rows, F, act, dz, ld_dz, h, ld_h))
        return rc;
    if (rows == 0)
        return ACSC_OK;
    const Epi e = epi_backward_act(z, ld_z, q_gate, q_up, act, dz, ld_dz, h, ld_h);
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>((rows * ((F + 511) / 512) + 3) / 4, 1 << 20)));
    if (dt == ACSC_BF16)
        ACSC_LAUNCH("glu_backward_act", glu_act_kernel<uint16_t>, grid, dim3(256), 0, stream, static_cast<const uint16_t *>(dh), ld_dh,
                    rows, F, e);
    else
        ACSC_LAUNCH("glu_backward_act", glu_act_kernel<float>, grid, dim3(256), 0, stream, static_cast<const float *>(dh), ld_dh, rows,
                    F, e);
    return check_launch("glu_backward_act");
}

extern "C" int glu_bias_workspace_size(int64_t rows, int F, size_t *bytes)
{
    clear_error();
    if (int rc = check_glu(rows, 1, F, ACSC_F32))
        return rc;
    ACSC_CHECK_ARG(bytes, ACSC_EINVAL, "null pointer to the result");
    *bytes = act_bytes(rows, F);
    return ACSC_OK;
}

extern "C" int glu_backward_act_bias(const void *dh, int64_t ld_dh, const void *z, int64_t ld_z, const q8_tensor *q_gate,
                                     const q8_tensor *q_up, acsc_dtype dt, int64_t rows, int F, acsc_act act, void *dz,
                                     int64_t ld_dz, void *h, int64_t ld_h, float *dbias, int accumulate, void *ws,
                                     size_t ws_bytes, hipStream_t stream)
{
    clear_error();
    if (int rc = check_backward_act(dh, ld_dh, z, ld_z, q_gate, q_up, dt, rows, F, act, dz, ld_dz, h, ld_h))
        return rc;
    ACSC_CHECK_ARG(dbias, ACSC_EINVAL, "null pointer dbias");
    ACSC_CHECK_ARG(aligned(dbias, 4), ACSC_EALIGN, "dbias not 4-byte aligned");
    if (rows == 0) {
        if (accumulate)
            return ACSC_OK;
        ACSC_LAUNCH("glu_zero", glu_zero_kernel, dim3((2 * F + 255) / 256), dim3(256), 0, stream, dbias, 2 * F);
        return check_launch("glu_zero");
    }
    const int parts = act_partials(rows, F);
    if (int rc = check_ws(ws, ws_bytes, act_bytes(rows, F)))
        return rc;
    // the sum over the partials takes them for rows of one tile each
    Gemm g{};
    g.N = F;
    g.tm = g.whole = parts;
    g.tn = 1;
    g.e = epi_backward_act(z, ld_z, q_gate, q_up, act, dz, ld_dz, h, ld_h);
    g.e.sums = parts > 1 ? static_cast<float *>(ws) : dbias;
    const int add = parts == 1 && accumulate;
    const dim3 grid((F + 511) / 512, parts);
    const int64_t per = (rows + parts - 1) / parts;
    if (dt == ACSC_BF16)
        ACSC_LAUNCH("glu_backward_act", glu_act_sums_kernel<uint16_t>, grid, dim3(256), 0, stream, static_cast<const uint16_t *>(dh),
                    ld_dh, rows, F, g.e, per, add);
    else
        ACSC_LAUNCH("glu_backward_act", glu_act_sums_kernel<float>, grid, dim3(256), 0, stream, static_cast<const float *>(dh), ld_dh,
                    rows, F, g.e, per, add);
    if (int rc = check_launch("glu_backward_act"))
        return rc;
    if (parts == 1)
        return ACSC_OK;
    ACSC_LAUNCH("glu_sums", glu_sums_kernel, dim3((2 * F + 63) / 64), dim3(64 * kSlices), 0, stream, g, F, dbias, accumulate);
    return check_launch("glu_sums");
}

extern "C" int glu_backward_input(const void *dy, int64_t ld_dy, acsc_dtype dt, int64_t rows, int F, int n_out, const void *W,
                                  int64_t ld_w, acsc_act act, const void *z, int64_t ld_z, const q8_tensor *q_gate,
                                  const q8_tensor *q_up, void *dz, int64_t ld_dz, void *h, int64_t ld_h, float *dbias, int accumulate,
                                  void *ws, size_t ws_bytes, hipStream_t stream)
{
    clear_error();
    if (int rc = check_glu(rows, n_out, F, dt))
        return rc;
    if (int rc = check_act(act))
        return rc;
    const bool some = rows > 0;
    if (int rc = check_mat(dy, some, ld_dy, n_out, dt, "dy"))
        return rc;
    if (int rc = check_mat(W, some, ld_w, F, dt, "W"))
        return rc;
    if (int rc = check_kept_pair(z, ld_z, q_gate, q_up, rows, F, dt))
        return rc;
    if (int rc = check_mat(dz, some, ld_dz, 2 * F, dt, "dz"))
        return rc;
    if (h)
        if (int rc = check_mat(h, some, ld_h, F, dt, "h"))
            return rc;
    ACSC_CHECK_ARG(!some || (dz != dy && dz != W && dz != h), ACSC_EINVAL, "dz must not overlap dy, W or h");
    ACSC_CHECK_ARG(!some || !h || (h != dy && h != W && h != z), ACSC_EINVAL, "h must not overlap dy, W or z");
    ACSC_CHECK_ARG(!some || dz != z || ld_dz == ld_z, ACSC_EINVAL, "dz in place of z needs ld_dz == ld_z");
    ACSC_CHECK_ARG(aligned(dbias, 4), ACSC_EALIGN, "dbias not 4-byte aligned");
    if (!some) {
        if (!dbias || accumulate)
            return ACSC_OK;
        ACSC_LAUNCH("glu_zero", glu_zero_kernel, dim3((2 * F + 255) / 256), dim3(256), 0, stream, dbias, 2 * F);
        return check_launch("glu_zero");
    }
    Gemm g{};
    g.A = {dy, ld_dy};
    g.B = {W, ld_w};
    const Shape s = shape_of(kGluGate, rows, F, n_out);
    const Plan p = plan_of(kGluGate, s, dt, readable(g.A, false, n_out, dt), readable(g.B, true, F, dt));
    if (int rc = check_tiles(p))
        return rc;
    const size_t sums = dbias ? sums_bytes(p, F) : 0;
    if (int rc = check_ws(ws, ws_bytes, sums + p.bytes()))
        return rc;
    g.e = Epi{dz, ld_dz, nullptr, nullptr, 0, const_cast<void *>(z), ld_z, q8_of(q_gate), act, 0, q8_of(q_up), h, ld_h,
              dbias ? static_cast<float *>(ws) : nullptr, cut_first(p), cut_slots(p)};
    if (int rc = run_product(g, kGluGate, p, s, dt, dt, static_cast<char *>(ws) + sums, nullptr, nullptr, stream, "glu_backward_input"))
        return rc;
    if (!dbias)
        return ACSC_OK;
    ACSC_LAUNCH("glu_sums", glu_sums_kernel, dim3((2 * F + 63) / 64), dim3(64 * kSlices), 0, stream, g, p.tile, dbias, accumulate);
    return check_launch("glu_sums");
}
