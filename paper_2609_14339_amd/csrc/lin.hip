// Linear layers: the entry points, how a product is cut, and the kernels
// before and after it.
#include "lin_plan.h"

namespace acsc {

namespace {

template <int KIND, typename TO>
__device__ __forceinline__ void join(const Gemm &g, const float *p, int64_t step, bool on, int64_t m, int n)
{
    const int left = on ? g.N - n : 0;
    float v[8] = {}, bias[8];
    if (left > 0)
        add_pieces(p, step, g.splits, v);
    load_bias<TO, KIND>(g.e, n, g.N, bias);
    Beside<TO> beside;
    if (has_beside<TO, KIND>(g.e))
        load_beside<TO, KIND>(g.e, beside, on ? m : 0, n, left);
    epilogue<TO, KIND>(g.e, v, bias, beside, m, n, left);
}
template <typename TO>
__global__ __launch_bounds__(256) void lin_join_few_kernel(Gemm g)
{
    const int64_t m = blockIdx.y;
    const int n = (blockIdx.x * 256 + threadIdx.x) * 8;
    join<kForward, TO>(g, g.part + m * g.ldp + n, g.M * g.ldp, true, m, n);
}
template <int KIND, typename TO, int TM, int T>
__global__ __launch_bounds__(256) void lin_join_kernel(Gemm g)
{
    // sixteen lanes at least to a row, a checkpoint's group of it
    constexpr int W = T < 128 ? 128 : T, PER = TM * W / 2048;
    const int64_t id = blockIdx.x / PER, count = static_cast<int64_t>(g.tm) * g.tn - g.whole;
    const int c = (blockIdx.x % PER) * 256 + threadIdx.x, row = c / (W / 8), col = c % (W / 8) * 8;
    int tile_m, tile_n;
    tile_at(g, g.whole + id, tile_m, tile_n);
    const int64_t m = static_cast<int64_t>(tile_m) * TM + row;
    join<KIND, TO>(g, g.part + (id * TM + row) * T + col, count * TM * T, m < g.M && col < T, m, tile_n * T + col);
}

// What a product needs done first, up to three jobs in one launch (a launch
// costs a small call 4 us): operands as the product reads them, and db.
struct Job {
    int db;              // 0: y <- act(x), or of a checkpoint's values, its rows filled with zeros up to a multiple
    const void *x;       // of eight; 1: column sums of x
    int64_t ldx, rows;
    int cols;
    void *y;             // job 1: db itself, or slices of it
    int64_t ldy;         // job 1: rows of a slice
    Q8 q;
    int act, accumulate;
    int blocks;          // workgroups of the job
    int across;          // job 1: workgroups along the columns
};
struct Jobs {
    int n;
    Job j[3];
};

// An operand: a wave takes 512 columns of a row, eight a lane.  An activation
// is rounded to T here, as the forward product's input was: dW of 8192 x 14336
// -> 4096 in bf16 is 2.3e-3 off with it and 1.7e-3, its own rounding, without;
// that would take its product in fp32 (by their rates 7.4 ms, 0.72 so) or
// twice, in two halves.  Sums: 512 columns and one slice of rows a workgroup,
// whose four waves take every fourth row and meet in LDS in order.
template <typename T>
__global__ __launch_bounds__(256) void lin_prepare_kernel(Jobs jobs)
{
    __shared__ float meet[4][512];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    int block = blockIdx.x, which = 0;
    while (which + 1 < jobs.n && block >= jobs.j[which].blocks) {
        block -= jobs.j[which].blocks;
        ++which;
    }
    const Job &j = jobs.j[which];
    const T *x = static_cast<const T *>(j.x);
    if (!j.db) {
        const int segs = (j.cols + 511) / 512;
        T *y = static_cast<T *>(j.y);
        for (int64_t w = static_cast<int64_t>(block) * 4 + wave; w < j.rows * segs; w += static_cast<int64_t>(j.blocks) * 4) {
            const int64_t row = w / segs;
            const int col = static_cast<int>(w - row * segs) * 512 + lane * 8;
            if (col >= j.cols)
                continue;
            float v[8];
            if (j.q.codes)
                load_codes(j.q.codes + row * j.q.ldc + col, j.cols - col, j.q.scales[row * j.q.lds + col / kGroup], v);
            else
                load8(x + row * j.ldx + col, j.cols - col, v);
            apply_act<T>(v, j.act);
            store8(y + row * j.ldy + col, 8, v);
        }
        return;
    }
    const int cb = block % j.across, sl = block / j.across, n = cb * 512 + lane * 8;
    const int64_t end = min<int64_t>(j.rows, (sl + static_cast<int64_t>(1)) * j.ldy);
    float s[8] = {};
#pragma unroll 8
    for (int64_t r = sl * j.ldy + wave; r < end; r += 4) {
        Raw8<T> v;
        load_raw(x + r * j.ldx + n, j.cols - n, v);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            s[i] += v.at(i);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        meet[wave][i * 64 + lane] = s[i];
    __syncthreads();
    const bool one = j.blocks == j.across;
    float *out = static_cast<float *>(j.y) + static_cast<int64_t>(sl) * j.cols;
    for (int c = threadIdx.x; c < 512; c += 256) {
        const int at = (c & 7) * 64 + (c >> 3), col = cb * 512 + c;
        if (col < j.cols) {
            const float v = ((meet[0][at] + meet[1][at]) + meet[2][at]) + meet[3][at];
            out[col] = one && j.accumulate ? out[col] + v : v;
        }
    }
}

// rows == 0: the weight gradients are sums over nothing.
template <typename TO>
__global__ __launch_bounds__(256) void lin_zero_kernel(TO *y, int64_t ldy, int64_t M, int N)
{
    const int n = blockIdx.x * 256 + threadIdx.x;
    if (n < N)
        for (int64_t m = blockIdx.y; m < M; m += gridDim.y)
            y[m * ldy + n] = 0;
}

// dz = dy act'(z): a wave takes 512 columns of a row, eight a lane.
template <typename T>
__global__ __launch_bounds__(256) void lin_act_kernel(const T *dy, int64_t lddy, const T *z, int64_t ldz, Q8 q, int64_t rows,
                                                      int N, int act, T *dz, int64_t lddz)
{
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int segs = (N + 511) / 512;
    for (int64_t w = static_cast<int64_t>(blockIdx.x) * 4 + wave; w < rows * segs; w += static_cast<int64_t>(gridDim.x) * 4) {
        const int64_t row = w / segs;
        const int col = static_cast<int>(w - row * segs) * 512 + lane * 8;
        if (col >= N)
            continue;
        float g[8], v[8];
        load8(dy + row * lddy + col, N - col, g);
        if (q.codes)
            load_codes(q.codes + row * q.ldc + col, N - col, q.scales[row * q.lds + col / kGroup], v);
        else
            load8(z + row * ldz + col, N - col, v);
        apply_slope<T>(g, v, act);
        store8(dz + row * lddz + col, N - col, g);
    }
}

// Tile and pieces of the sum, by the least estimated time.  A round is what
// the card runs at once, `at_once` workgroups a CU.  Whole rounds of tiles are
// not cut; the tiles of a last, partial one may be, so that their pieces fill
// the card.  The times are measured: a 256 tile takes 1.5 us a step of 64 and
// 5 beside them (bf16 4096 x 2048 -> 8192: 56 a round of 32 steps); a bf16 128
// tile 1.0 and 3 with a second one on its CU (2048 x 2048 -> 8192: 34.5 a
// round), 0.65 alone; an fp32 tile 4.1 a step of 32 (130 TFLOP/s at 4096^3),
// 2.2 alone; the narrow tiles wait for W's bytes from memory, and 4096 ->
// 14336 alone took 0.9 (bf16) and 1.2 (fp32); the pieces' sum 10 for waiting
// and the launch, and their bytes, written and read, at 4.5 TB/s.
// Both sides: 2048 x 2048 -> 8192 in 256 tiles of two pieces each 99 us, in
// whole 128 tiles 58; the tiles of the last round cut or not, 15057 x 3904 ->
// 1216 144 or 163, input gradient of 1198 x 13312 -> 2176 81 or 93, 3000 x 3000
// -> 3000 (not chosen) 88 or 80; 4096 -> 14336, forward / input gradient of 12,
// 52, 128 tokens: tiles of 32 rows bf16 29/31, 57/39, 63/57, fp32 -/56, 86/87,
// 207/139; of 64 31/37, 31/38, 60/44, -/78, 84/83, 151/137; of 128 44/40, 46/41,
// 46/46, -/136, 147/131, 143/137.  The gated product's gradient: whole tiles wait for their epilogue, the
// pieces' sum has it spread over the card (128 x 4096 -> 14336: 63 us in whole
// tiles of 128 x 64, 41 in two pieces of 128 x 128).  Against each tile alone
// on twelve shapes of 256 to 14455 rows the choice is within 4% of the best.
struct Cut {
    int rows, tile, whole, splits, per;
};
struct Tile {
    int rows, cols;
    int at_once;          // workgroups of a CU
    double step, alone;   // us of a step with as many, and with one
    double edge;
    double gated;         // more beside them with the gated product's gradient in the epilogue
};
// codes: a gated product's pre-activations are coded, whose groups lie in two
// tiles of 128 columns each: there every tile goes through the pieces' sum.
inline Cut cut_of(EpiKind kind, const Shape &s, int steps, bool bf16, bool codes)
{
    static const Tile kBf16[] = {
        {256, 256, 1, 1.5, 1.5, 5, 20}, {128, 128, 2, 1.0, 0.65, 3, 9}, {64, 128, 3, 1.05, 0.85, 3, 6}, {32, 128, 4, 1.0, 0.8, 3, 4}, {128, 64, 2, 0.8, 0.55, 3, 12}};
    static const Tile kF32[] = {{128, 128, 2, 4.1, 2.2, 3, 9}, {64, 128, 3, 3.2, 1.2, 3, 6}, {32, 128, 4, 2.3, 1.2, 3, 4}, {128, 64, 2, 2.2, 1.2, 3, 12}};
    const Tile *first = bf16 ? kBf16 : kF32, *end = bf16 ? std::end(kBf16) : std::end(kF32);
    Cut best{};
    double least = 0;
    for (const Tile *t = first; t != end; ++t) {
        // 32 rows of a col operand are not a whole block of it in LDS; 64
        // columns would split the group of a checkpoint that is written
        if ((t->rows == 32 && kind == kWeight) || (t->cols == 64 && (kind == kGluForward || (kind == kForward && s.N > 64))))
            continue;
        const int64_t tiles = ((s.M + t->rows - 1) / t->rows) * ((s.N + t->cols - 1) / t->cols);
        const int slots = 256 * t->at_once;
        const auto rounds = [&](int64_t groups, int per, bool whole) {
            const double edge = t->edge + (whole && kind == kGluGate ? t->gated : 0);
            const int64_t rest = groups % slots, beside = (rest + 255) / 256 - 1;
            const double step = t->at_once > 1 ? t->alone + (t->step - t->alone) * static_cast<double>(beside) / (t->at_once - 1) : t->alone;
            return static_cast<double>(groups / slots) * (per * t->step + edge) + (rest ? per * step + edge : 0);
        };
        const bool all = codes && kind == kGluForward && t->cols == 128;   // through the pieces' sum
        const int64_t rest = all ? tiles : tiles % slots;
        for (int want = 1; want == 1 || (rest && want <= 64 && steps / want >= 4 && rest * want <= 2048);
             want += want < 8 ? 1 : 8) {
            const int per = (steps + want - 1) / want, n = (steps + per - 1) / per;
            const double us = n == 1 && !all ? rounds(tiles, steps, true)
                                     : rounds(tiles - rest, steps, true) + rounds(rest * n, per, false) + 10 +
                                           n * static_cast<double>(rest) * t->rows * t->cols * 8 / 4.5e6;
            if (least == 0 || us < least) {
                least = us;
                best = Cut{t->rows, t->cols, static_cast<int>(n == 1 && !all ? tiles : tiles - rest), n, per};
            }
        }
    }
    return best;
}

// The most that the pieces of a coded product's tiles take at a time (more only
// where one row of tiles does): all of its pre-activations go through them, and
// whole they would take the memory that the 8 bits are to save.  fp32 16384 x
// 2048 -> 8192 7815 us in four runs, 7765 in one with 1 GiB, 7530 without codes;
// 40003 x 24 -> 1030 224 in two, whose pieces stay in the caches, 258 in one.
constexpr size_t kCodedPieces = static_cast<size_t>(256) << 20;

}  // namespace

Plan plan_of(EpiKind kind, const Shape &s, acsc_dtype dt, bool fits_a, bool fits_b, bool codes)
{
    Plan p{};
    const bool bf16 = dt == ACSC_BF16;
    const int bk = 128 / static_cast<int>(dtype_size(dt));
    const int64_t K = s.K;   // up to 2^31 - 1 rows: what rounds it up takes 64 bits
    const int steps = static_cast<int>((K + bk - 1) / bk);
    if (kind == kWeight && s.K <= few_tokens(kind, fits_b)) {
        p.few = true;
        p.splits = 1;
        return p;
    }
    if ((kind == kForward || kind == kGluForward) && s.M <= few_tokens(kind, fits_b)) {
        // 16 outputs (or eight of each kind) a workgroup: a cut only where they fill half the CUs at
        // most, at two rounds of eight lines a piece
        const int cols = kind == kGluForward ? s.N / 2 : s.N, groups = kind == kGluForward ? (cols + 7) / 8 : (cols + 15) / 16;
        const int round = 8 * 128 / static_cast<int>(dtype_size(dt)), rounds = (s.K + round - 1) / round;
        const int want = groups >= 128 ? 1 : std::max(1, std::min((255 + groups) / groups, rounds / 2));
        const int per = (rounds + want - 1) / want;
        p.few = true;
        p.splits = (rounds + per - 1) / per;
        p.kchunk = per * round;
        p.ldp = up8(cols);
        p.part = up256(static_cast<size_t>(p.splits) * s.M * p.ldp * 4 * (s.N / cols));
        return p;
    }
    const Cut c = cut_of(kind, s, steps, bf16, codes);
    p.rows = c.rows;
    p.tile = c.tile;
    p.tm = static_cast<int>((s.M + p.rows - 1) / p.rows);
    p.tn = (s.N + p.tile - 1) / p.tile;
    p.whole = c.whole;
    p.splits = c.splits;
    p.kchunk = static_cast<int>(std::min(K, static_cast<int64_t>(c.per) * bk));
    p.part = up256(static_cast<size_t>(static_cast<int64_t>(p.tm) * p.tn - p.whole) * p.splits * p.rows * p.tile * 4);
    if (kind == kWeight) {
        // db's slices of at least 32 rows, up to about two workgroups a CU
        const int64_t blocks = (s.M + 511) / 512;
        p.slices = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(512 / blocks, K / 32)));
        p.slice = static_cast<int>((K + p.slices - 1) / p.slices);
        p.slices = static_cast<int>((K + p.slice - 1) / p.slice);
        p.db = p.slices > 1 ? up256(static_cast<size_t>(p.slices) * s.M * 4) : 0;
    }
    const int64_t es = static_cast<int64_t>(dtype_size(dt));
    p.pack_a = !fits_a;
    p.pack_b = !fits_b;
    p.lda = up8(s.acol ? static_cast<int>(s.M) : s.K);
    p.ldb = up8(s.bcol ? s.N : s.K);
    p.a = p.pack_a ? up256(static_cast<size_t>(s.acol ? s.K : s.M) * p.lda * es) : 0;
    p.b = p.pack_b ? up256(static_cast<size_t>(s.bcol ? s.K : s.N) * p.ldb * es) : 0;
    p.band = p.tm;
    if (codes && kind == kGluForward && p.tile == 128 && p.part > kCodedPieces) {
        // runs of as many rows of tiles each as fit, and as even as they can be
        const size_t row = static_cast<size_t>(p.tn) * p.splits * p.rows * p.tile * 4;
        const int fit = static_cast<int>(std::max<size_t>(1, kCodedPieces / row)), runs = (p.tm + fit - 1) / fit;
        p.band = (p.tm + runs - 1) / runs;
        p.part = up256(p.band * row);
        p.a = p.pack_a ? up256(static_cast<size_t>(p.band) * p.rows * p.lda * es) : 0;
    }
    return p;
}

namespace {

template <int KIND, typename TO>
void launch_join(const Gemm &g, const Plan &p, hipStream_t st)
{
    const int tail = p.tm * p.tn - p.whole;
    const dim3 grid(tail * (p.rows * std::max(p.tile, 128) / 2048));
    if (p.rows == 256) {
        ACSC_LAUNCH("lin_join", (lin_join_kernel<KIND, TO, 256, 256>), grid, dim3(256), 0, st, g);
        return;
    }
    if (p.rows == 64) {
        ACSC_LAUNCH("lin_join", (lin_join_kernel<KIND, TO, 64, 128>), grid, dim3(256), 0, st, g);
        return;
    }
    if (p.tile == 64) {
        ACSC_LAUNCH("lin_join", (lin_join_kernel<KIND, TO, 128, 64>), grid, dim3(256), 0, st, g);
        return;
    }
    if constexpr (KIND != kWeight)
        if (p.rows == 32) {
            ACSC_LAUNCH("lin_join", (lin_join_kernel<KIND, TO, 32, 128>), grid, dim3(256), 0, st, g);
            return;
        }
    ACSC_LAUNCH("lin_join", (lin_join_kernel<KIND, TO, 128, 128>), grid, dim3(256), 0, st, g);
}

inline void add_operand(Jobs &jobs, const Operand &from, int64_t rows, int cols, void *to, int64_t ld, const Kept &kept)
{
    Job &j = jobs.j[jobs.n++];
    j.x = from.p;
    j.ldx = from.ld;
    j.rows = rows;
    j.cols = cols;
    j.y = to;
    j.ldy = ld;
    j.q = kept.q;
    j.act = kept.act;
    j.blocks = static_cast<int>(std::min<int64_t>((rows * ((cols + 511) / 512) + 3) / 4, 1 << 18));
}

}  // namespace

// What comes first, the product and its pieces' sum; `out` is the type of the
// output.
int run_product(Gemm &g, EpiKind kind, const Plan &p, const Shape &s, acsc_dtype dt, acsc_dtype out, char *ws, float *db,
                const Again *again, hipStream_t st, const char *tag)
{
    g.M = s.M;
    g.N = kind == kGluForward ? s.N / 2 : s.N;
    g.K = s.K;
    g.tm = p.tm;
    g.tn = p.tn;
    g.splits = p.splits;
    g.kchunk = p.kchunk;
    g.ldp = p.ldp;
    g.whole = p.whole;
    const int chunk = 16 / static_cast<int>(dtype_size(dt));
    g.words_a = !p.pack_a && (s.acol ? s.M : s.K) % chunk;
    g.words_b = !p.pack_b && !again && (s.bcol ? s.N : s.K) % chunk;
    // a piece goes through memory if there are more, or if the workgroups of a
    // product for few tokens, or of narrow tiles of a gated one, hold no whole
    // checkpoint groups
    const bool pieces = p.splits > 1 || (g.e.q.codes && (p.few || (kind == kGluForward && p.tile == 128)));
    g.part = pieces ? reinterpret_cast<float *>(ws) : nullptr;
    Jobs jobs{};
    if (again)
        add_operand(jobs, again->from, s.K, s.N, again->to, up8(s.N), again->kept);
    if (db) {
        Job &j = jobs.j[jobs.n++];
        j.db = 1;
        j.x = g.A.p;
        j.ldx = g.A.ld;
        j.rows = s.K;
        j.cols = static_cast<int>(s.M);
        j.accumulate = g.e.accumulate;
        j.across = static_cast<int>((s.M + 511) / 512);
        j.blocks = j.across * p.slices;
        j.ldy = p.slice;
        j.y = p.slices > 1 ? static_cast<void *>(ws + p.part) : db;
        if (p.slices > 1) {
            g.dbpart = reinterpret_cast<float *>(ws + p.part);
            g.slices = p.slices;
            g.db = db;
        }
    }
    char *copy = ws + p.part + p.db;
    const Kept plain{q8_of(nullptr), ACSC_ACT_NONE};
    if (p.pack_a) {
        add_operand(jobs, g.A, s.acol ? s.K : s.M, s.acol ? static_cast<int>(s.M) : s.K, copy, p.lda, plain);
        g.A = {copy, p.lda};
        copy += p.a;
    }
    if (p.pack_b) {
        add_operand(jobs, g.B, s.bcol ? s.K : s.N, s.bcol ? s.N : s.K, copy, p.ldb, plain);
        g.B = {copy, p.ldb};
    }
    if (jobs.n) {
        int blocks = 0;
        for (int i = 0; i < jobs.n; ++i)
            blocks += jobs.j[i].blocks;
        if (dt == ACSC_BF16)
            ACSC_LAUNCH("lin_prepare", lin_prepare_kernel<uint16_t>, dim3(blocks), dim3(256), 0, st, jobs);
        else
            ACSC_LAUNCH("lin_prepare", lin_prepare_kernel<float>, dim3(blocks), dim3(256), 0, st, jobs);
        if (int rc = check_launch("lin_prepare"))
            return rc;
    }
    if (p.few) {
        if (int rc = kind == kGluForward ? glu_few_run(g, dt, st, tag) : lin_few_run(g, dt, st, tag))
            return rc;
    } else if (int rc = kind >= kGluForward ? glu_tile_run(g, p.rows, p.tile, kind, dt, st, tag)
                                            : lin_tile_run(g, p.rows, p.tile, kind, dt, out, st, tag)) {
        return rc;
    }
    if (pieces) {
        const bool b = out == ACSC_BF16;
        if (kind >= kGluForward) {
            glu_join_run(g, p, kind, dt, st);
        } else if (p.few) {
            const dim3 grid((g.N + 2047) / 2048, static_cast<unsigned>(g.M));
            if (b)
                ACSC_LAUNCH("lin_join", lin_join_few_kernel<uint16_t>, grid, dim3(256), 0, st, g);
            else
                ACSC_LAUNCH("lin_join", lin_join_few_kernel<float>, grid, dim3(256), 0, st, g);
        } else if (kind == kForward) {
            b ? launch_join<kForward, uint16_t>(g, p, st) : launch_join<kForward, float>(g, p, st);
        } else if (kind == kGate) {
            b ? launch_join<kGate, uint16_t>(g, p, st) : launch_join<kGate, float>(g, p, st);
        } else {
            b ? launch_join<kWeight, uint16_t>(g, p, st) : launch_join<kWeight, float>(g, p, st);
        }
        if (int rc = check_launch("lin_join"))
            return rc;
    }
    return ACSC_OK;
}

namespace {

// Bytes of an activation recomputed for the weight gradient.
inline size_t recomputed_bytes(int64_t rows, int n_in, acsc_dtype dt)
{
    return up256(static_cast<size_t>(rows) * ((n_in + 7) / 8 * 8) * dtype_size(dt));
}

}  // namespace
}  // namespace acsc

using namespace acsc;

static int check_product(lin_op op, int64_t rows, int n_in, int n_out, acsc_dtype dt, const void *out)
{
    if (int rc = check_layer(rows, n_in, n_out, dt))
        return rc;
    ACSC_CHECK_ARG(out, ACSC_EINVAL, "null pointer to the result");
    ACSC_CHECK_ARG(op == LIN_FORWARD || op == LIN_BACKWARD_INPUT || op == LIN_BACKWARD_WEIGHT, ACSC_EINVAL,
                   "unknown product %d", (int)op);
    return ACSC_OK;
}

// The plan of a product, with the operands' copies that bits 0 (A) and 1 (B) of
// `copies` add to those that are needed whatever the alignment.
static int plan_product(lin_op op, int64_t rows, int n_in, int n_out, acsc_dtype dt, int copies, Plan &p)
{
    const EpiKind kind = op == LIN_FORWARD ? kForward : op == LIN_BACKWARD_INPUT ? kGate : kWeight;
    const Shape s = shape_of(kind, rows, n_in, n_out);
    // the strides that the plan is good for: all from the rows' own length on, of whole words
    const auto best = [&](bool col, int64_t inner) {
        return readable(Operand{nullptr, dt == ACSC_F32 ? inner : (inner + 1) / 2 * 2}, col, inner, dt);
    };
    const bool a = best(s.acol, s.acol ? s.M : s.K), b = best(s.bcol, s.bcol ? s.N : s.K);
    p = plan_of(kind, s, dt, a && !(copies & 1), b && !(copies & 2));
    return check_tiles(p);
}

static int workspace_size(lin_op op, int64_t rows, int n_in, int n_out, acsc_dtype dt, bool any, size_t *bytes)
{
    clear_error();
    if (int rc = check_product(op, rows, n_in, n_out, dt, bytes))
        return rc;
    *bytes = 0;
    if (rows == 0)
        return ACSC_OK;
    // with any alignment: the most that either operand's copy, or its absence, takes
    size_t most = 0;
    for (int copies = 0; copies < (any ? 4 : 1); ++copies) {
        Plan p;
        if (int rc = plan_product(op, rows, n_in, n_out, dt, copies, p))
            return rc;
        most = std::max(most, p.bytes());
    }
    *bytes = most;
    if (op == LIN_BACKWARD_WEIGHT && rows > few_tokens(kWeight, true))
        *bytes += recomputed_bytes(rows, n_in, dt);
    return ACSC_OK;
}

extern "C" int lin_product_plan(lin_op op, int64_t rows, int n_in, int n_out, acsc_dtype dt, lin_plan *plan)
{
    clear_error();
    if (int rc = check_product(op, rows, n_in, n_out, dt, plan))
        return rc;
    *plan = lin_plan{};
    if (rows == 0)
        return ACSC_OK;
    Plan p;
    if (int rc = plan_product(op, rows, n_in, n_out, dt, 0, p))
        return rc;
    *plan = {p.rows, p.tile, p.whole, static_cast<int64_t>(p.tm) * p.tn - p.whole, p.splits};
    return ACSC_OK;
}

extern "C" int lin_workspace_size(lin_op op, int64_t rows, int n_in, int n_out, acsc_dtype dt, size_t *bytes)
{
    return workspace_size(op, rows, n_in, n_out, dt, false, bytes);
}

extern "C" int lin_workspace_size_unaligned(lin_op op, int64_t rows, int n_in, int n_out, acsc_dtype dt, size_t *bytes)
{
    return workspace_size(op, rows, n_in, n_out, dt, true, bytes);
}

extern "C" int lin_forward(const void *x, int64_t ld_x, acsc_dtype dt, int64_t rows, int n_in, int n_out, const void *W,
                           int64_t ld_w, const void *bias, acsc_act act, const void *residual, int64_t ld_res, void *y,
                           int64_t ld_y, void *z, int64_t ld_z, const q8_tensor *q, void *ws, size_t ws_bytes,
                           hipStream_t stream)
{
    clear_error();
    if (int rc = check_layer(rows, n_in, n_out, dt))
        return rc;
    if (int rc = check_act(act))
        return rc;
    const bool some = rows > 0;
    if (int rc = check_mat(x, some, ld_x, n_in, dt, "x"))
        return rc;
    if (int rc = check_mat(W, some, ld_w, n_in, dt, "W"))
        return rc;
    if (int rc = check_mat(y, some, ld_y, n_out, dt, "y"))
        return rc;
    ACSC_CHECK_ARG(aligned(bias, dtype_size(dt)), ACSC_EALIGN, "bias not aligned to its elements");
    if (residual)
        if (int rc = check_mat(residual, some, ld_res, n_out, dt, "residual"))
            return rc;
    ACSC_CHECK_ARG(residual != y || !some || ld_res == ld_y, ACSC_EINVAL, "y in place of the residual needs ld_y == ld_res");
    ACSC_CHECK_ARG(!some || (y != x && y != W && y != z), ACSC_EINVAL, "y must not overlap x, W or z");
    if (z)
        if (int rc = check_mat(z, some, ld_z, n_out, dt, "z"))
            return rc;
    ACSC_CHECK_ARG(!some || !z || (z != x && z != W), ACSC_EINVAL, "z must not overlap x or W");
    if (q)
        if (int rc = check_q8(q, rows, n_out))
            return rc;
    if (!some)
        return ACSC_OK;
    Gemm g{};
    g.A = {x, ld_x};
    g.B = {W, ld_w};
    const Shape s = shape_of(kForward, rows, n_in, n_out);
    const Plan p = plan_of(kForward, s, dt, readable(g.A, false, n_in, dt), readable(g.B, false, n_in, dt));
    if (int rc = check_tiles(p))
        return rc;
    if (int rc = check_ws(ws, ws_bytes, p.bytes()))
        return rc;
    g.e = Epi{y, ld_y, bias, residual, ld_res, z, ld_z, q8_of(q), act, 0};
    return run_product(g, kForward, p, s, dt, dt, static_cast<char *>(ws), nullptr, nullptr, stream, "lin_forward");
}

extern "C" int lin_backward_act(const void *dy, int64_t ld_dy, const void *z, int64_t ld_z, const q8_tensor *q,
                                acsc_dtype dt, int64_t rows, int n_out, acsc_act act, void *dz, int64_t ld_dz,
                                hipStream_t stream)
{
    clear_error();
    if (int rc = check_layer(rows, 1, n_out, dt))
        return rc;
    if (int rc = check_act(act))
        return rc;
    if (int rc = check_mat(dy, rows > 0, ld_dy, n_out, dt, "dy"))
        return rc;
    if (int rc = check_kept(z, ld_z, q, rows, n_out, dt))
        return rc;
    if (int rc = check_mat(dz, rows > 0, ld_dz, n_out, dt, "dz"))
        return rc;
    ACSC_CHECK_ARG(dz != dy || rows == 0 || ld_dz == ld_dy, ACSC_EINVAL, "dz in place of dy needs ld_dz == ld_dy");
    ACSC_CHECK_ARG(dz != z || rows == 0 || ld_dz == ld_z, ACSC_EINVAL, "dz in place of z needs ld_dz == ld_z");
    if (rows == 0)
        return ACSC_OK;
    const int64_t blocks = std::min<int64_t>((rows * ((n_out + 511) / 512) + 3) / 4, 1 << 20);
    if (dt == ACSC_BF16)
        ACSC_LAUNCH("lin_backward_act", lin_act_kernel<uint16_t>, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, stream,
                    static_cast<const uint16_t *>(dy), ld_dy, static_cast<const uint16_t *>(z), ld_z, q8_of(q), rows, n_out,
                    act, static_cast<uint16_t *>(dz), ld_dz);
    else
        ACSC_LAUNCH("lin_backward_act", lin_act_kernel<float>, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, stream,
                    static_cast<const float *>(dy), ld_dy, static_cast<const float *>(z), ld_z, q8_of(q), rows, n_out, act,
                    static_cast<float *>(dz), ld_dz);
    return check_launch("lin_backward_act");
}

extern "C" int lin_backward_input(const void *dz, int64_t ld_dz, acsc_dtype dt, int64_t rows, int n_in, int n_out,
                                  const void *W, int64_t ld_w, acsc_act act, const void *z, int64_t ld_z,
                                  const q8_tensor *q, void *dx, int64_t ld_dx, void *ws, size_t ws_bytes,
                                  hipStream_t stream)
{
    clear_error();
    if (int rc = check_layer(rows, n_in, n_out, dt))
        return rc;
    if (int rc = check_act(act))
        return rc;
    const bool some = rows > 0;
    if (int rc = check_mat(dz, some, ld_dz, n_out, dt, "dz"))
        return rc;
    if (int rc = check_mat(W, some, ld_w, n_in, dt, "W"))
        return rc;
    if (act != ACSC_ACT_NONE)
        if (int rc = check_kept(z, ld_z, q, rows, n_in, dt))
            return rc;
    if (int rc = check_mat(dx, some, ld_dx, n_in, dt, "dx"))
        return rc;
    ACSC_CHECK_ARG(!some || (dx != dz && dx != W), ACSC_EINVAL, "dx must not overlap dz or W");
    ACSC_CHECK_ARG(!some || act == ACSC_ACT_NONE || dx != z || ld_dx == ld_z, ACSC_EINVAL, "dx in place of z needs ld_dx == ld_z");
    if (!some)
        return ACSC_OK;
    Gemm g{};
    g.A = {dz, ld_dz};
    g.B = {W, ld_w};
    const Shape s = shape_of(kGate, rows, n_in, n_out);
    const Plan p = plan_of(kGate, s, dt, readable(g.A, false, n_out, dt), readable(g.B, true, n_in, dt));
    if (int rc = check_tiles(p))
        return rc;
    if (int rc = check_ws(ws, ws_bytes, p.bytes()))
        return rc;
    g.e = Epi{dx, ld_dx, nullptr, nullptr, 0, const_cast<void *>(z), ld_z, q8_of(q), act, 0};
    return run_product(g, kGate, p, s, dt, dt, static_cast<char *>(ws), nullptr, nullptr, stream, "lin_backward_input");
}

extern "C" int lin_backward_weight(const void *dz, int64_t ld_dz, const void *x, int64_t ld_x, const q8_tensor *q,
                                   acsc_act act, acsc_dtype dt, int64_t rows, int n_in, int n_out, void *dW,
                                   acsc_dtype dw_dt, int64_t ld_dw, float *db, int accumulate, void *ws,
                                   size_t ws_bytes, hipStream_t stream)
{
    clear_error();
    if (int rc = check_layer(rows, n_in, n_out, dt))
        return rc;
    ACSC_CHECK_ARG(dw_dt == ACSC_F32 || dw_dt == ACSC_BF16, ACSC_EDTYPE, "unknown dtype %d of dW", (int)dw_dt);
    if (int rc = check_act(act))
        return rc;
    const bool some = rows > 0;
    if (int rc = check_mat(dz, some, ld_dz, n_out, dt, "dz"))
        return rc;
    if (int rc = check_kept(x, ld_x, q, rows, n_in, dt))
        return rc;
    if (int rc = check_mat(dW, true, ld_dw, n_in, dw_dt, "dW"))
        return rc;
    ACSC_CHECK_ARG(!some || (dW != dz && dW != x), ACSC_EINVAL, "dW must not overlap dz or x");
    ACSC_CHECK_ARG(aligned(db, 4), ACSC_EALIGN, "db not 4-byte aligned");
    if (!some) {
        if (accumulate)
            return ACSC_OK;
        const dim3 grid((n_in + 255) / 256, std::min(n_out, 65535));
        if (dw_dt == ACSC_BF16)
            ACSC_LAUNCH("lin_zero", lin_zero_kernel<uint16_t>, grid, dim3(256), 0, stream, static_cast<uint16_t *>(dW), ld_dw,
                        static_cast<int64_t>(n_out), n_in);
        else
            ACSC_LAUNCH("lin_zero", lin_zero_kernel<float>, grid, dim3(256), 0, stream, static_cast<float *>(dW), ld_dw,
                        static_cast<int64_t>(n_out), n_in);
        if (db)
            ACSC_LAUNCH("lin_zero", lin_zero_kernel<float>, dim3((n_out + 255) / 256, 1), dim3(256), 0, stream, db, 0,
                        static_cast<int64_t>(1), n_out);
        return check_launch("lin_zero");
    }
    // Few tokens: from what was kept, in one kernel.  Otherwise
    // the activation, or the checkpoint's values, whole: read once here, and
    // by the product many times.  Its rows end at a multiple of eight, so the
    // product reads it where it is.
    const Shape s = shape_of(kWeight, rows, n_in, n_out);
    Gemm g{};
    g.e = Epi{dW, ld_dw, nullptr, nullptr, 0, nullptr, 0, q8_of(nullptr), ACSC_ACT_NONE, accumulate};
    if (rows <= few_tokens(kWeight, true)) {
        g.A = {dz, ld_dz};
        g.B = {x, ld_x};
        g.M = s.M;
        g.N = s.N;
        g.K = s.K;
        return lin_few_weight_run(g, Kept{q8_of(q), act}, dt, dw_dt, db, stream, "lin_backward_weight");
    }
    const bool again = q || act != ACSC_ACT_NONE;
    const size_t whole = again ? recomputed_bytes(rows, n_in, dt) : 0;
    g.A = {dz, ld_dz};
    g.B = again ? Operand{ws, up8(n_in)} : Operand{x, ld_x};
    const Plan p = plan_of(kWeight, s, dt, readable(g.A, true, n_out, dt), again || readable(g.B, true, n_in, dt));
    if (int rc = check_tiles(p))
        return rc;
    if (int rc = check_ws(ws, ws_bytes, p.bytes() + whole))
        return rc;
    const Again a{{x, ld_x}, ws, Kept{q8_of(q), act}};
    return run_product(g, kWeight, p, s, dt, dw_dt, static_cast<char *>(ws) + whole, db, again ? &a : nullptr, stream,
                       "lin_backward_weight");
}
