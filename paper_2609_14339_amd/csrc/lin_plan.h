// How a linear layer's product is cut, what comes before and after it, and the
// checks of its arguments: what the plain and the gated entry points share.
#pragma once

#include "lin.h"

namespace acsc {

// Tokens up to which a product does without tiles.  Forward: W is read once
// and unstaged; 4096 -> 14336, 1 / 8 / 16 tokens, us: bf16 24, 28, 35 against 31
// by tiles for 4 to 64; fp32 53, 60, 68 against 56.  Where the tile kernel
// cannot read W it has to be copied first, three times its bytes: there the
// kernel is used as far as it goes.  Weight gradient: outer products of
// unrounded activations; bf16 8192 -> 8192, 1 / 4 / 8 tokens: 25.6, 30.0, 38.8
// against 43 by tiles.  (The input gradient by vector FMAs on rows of W read
// once took 39 against 31 by tiles.)
inline int few_tokens(EpiKind kind, bool fits_b)
{
    return kind == kForward || kind == kGluForward ? (fits_b ? 8 : 16) : kind == kWeight ? 8 : 0;
}

inline size_t up256(size_t b) { return (b + 255) / 256 * 256; }

// How a product is cut, and what of the workspace it takes: the pieces, db's
// pieces, and copies of the operands that the tile kernel cannot read where
// they are.
struct Plan {
    bool few;                               // the product for few tokens
    int rows, tile;                         // of a tile: its rows and columns
    int tm, tn, whole, splits, kchunk;
    int band;                               // rows of tiles of a run: all, or of a coded product as its pieces fit
    int slices, slice;                      // of the rows, for db
    int64_t ldp;
    bool pack_a, pack_b;
    int64_t lda, ldb;                       // row strides of the copies
    size_t part, db, a, b;                  // bytes
    size_t bytes() const { return part + db + a + b; }
};

inline int up8(int n) { return (n + 7) / 8 * 8; }

// A row operand keeps the sum's index in its rows, a col operand its own.
struct Shape {
    int64_t M;
    int N, K;
    bool acol, bcol;
};
inline Shape shape_of(EpiKind kind, int64_t rows, int n_in, int n_out)
{
    if (kind == kForward)
        return {rows, n_out, n_in, false, false};
    if (kind == kGluForward)
        return {rows, 2 * n_out, n_in, false, false};
    if (kind == kGate || kind == kGluGate)
        return {rows, n_in, n_out, false, true};
    return {n_out, n_in, static_cast<int>(rows), true, true};
}

// Whether the tile kernel reads an operand where it is: rows at multiples of
// the word that the DMA reads, rows of whole words, of a chunk at least if a
// col operand's last chunk runs on into the next row, and offsets within a
// tile and step of under 2^31 bytes.  Both sides, bf16 rows at odd words
// copied first or read there, us: 20 x 4098 -> 14338 67 and 29, 8190 x 8190 ->
// 8190 907 and 890, its input gradient 899 and 813.
inline bool readable(const Operand &o, bool col, int64_t inner, acsc_dtype dt)
{
    const int es = static_cast<int>(dtype_size(dt)), chunk = 16 / es, unit = 4 / es;
    return aligned(o.p, unit * es) && o.ld % unit == 0 && inner * es % 4 == 0 && (!col || inner % chunk == 0 || o.ld >= chunk) &&
           o.ld * es * (col ? 64 : 256) < (1ll << 31);
}

// An input of the weight gradient that is formed again from what was kept.
struct Again {
    Operand from;
    void *to;
    Kept kept;
};

// The plan of a product (codes: it writes an 8-bit checkpoint), and its run:
// what comes first, the product and its pieces' sum; `out` is the type of the
// output.
Plan plan_of(EpiKind kind, const Shape &s, acsc_dtype dt, bool fits_a, bool fits_b, bool codes = false);
int run_product(Gemm &g, EpiKind kind, const Plan &p, const Shape &s, acsc_dtype dt, acsc_dtype out, char *ws, float *db,
                const Again *again, hipStream_t st, const char *tag);

int lin_few_run(const Gemm &g, acsc_dtype dt, hipStream_t st, const char *tag);
int lin_few_weight_run(const Gemm &g, const Kept &kept, acsc_dtype dt, acsc_dtype out, float *db, hipStream_t st,
                       const char *tag);
int lin_tile_run(const Gemm &g, int rows, int cols, EpiKind kind, acsc_dtype dt, acsc_dtype out, hipStream_t st,
                 const char *tag);
int glu_few_run(const Gemm &g, acsc_dtype dt, hipStream_t st, const char *tag);
int glu_tile_run(const Gemm &g, int rows, int cols, EpiKind kind, acsc_dtype dt, hipStream_t st, const char *tag);
void glu_join_run(const Gemm &g, const Plan &p, EpiKind kind, acsc_dtype dt, hipStream_t st);

// Adds the pieces of a cut product in order and takes the sum through the
// epilogue, eight columns a thread: of few tokens, 2048 columns of a row a
// workgroup; of tiles, 2048 elements of a tile.
__device__ __forceinline__ void add_pieces(const float *p, int64_t step, int splits, float (&v)[8])
{
    const f32x4 *q = reinterpret_cast<const f32x4 *>(p);
    f32x4 lo = q[0], hi = q[1];
#pragma unroll 4
    for (int i = 1; i < splits; ++i) {
        lo += q[i * step / 4];
        hi += q[i * step / 4 + 1];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = lo[i];
        v[4 + i] = hi[i];
    }
}
inline int check_layer(int64_t rows, int n_in, int n_out, int dt)
{
    ACSC_CHECK_ARG(dt == ACSC_F32 || dt == ACSC_BF16, ACSC_EDTYPE, "unknown dtype %d", dt);
    ACSC_CHECK_ARG(rows >= 0 && rows < (1ll << 31), ACSC_EINVAL, "rows=%lld outside [0, 2^31)", (long long)rows);
    ACSC_CHECK_ARG(n_in >= 1 && n_in <= (1 << 22), ACSC_EINVAL, "n_in=%d outside [1, 2^22]", n_in);
    ACSC_CHECK_ARG(n_out >= 1 && n_out <= (1 << 22), ACSC_EINVAL, "n_out=%d outside [1, 2^22]", n_out);
    return ACSC_OK;
}

inline int check_mat(const void *p, bool need, int64_t ld, int cols, int dt, const char *name)
{
    ACSC_CHECK_ARG(!need || p, ACSC_EINVAL, "null pointer %s", name);
    ACSC_CHECK_ARG(ld >= cols && ld < (1ll << 40), ACSC_EINVAL, "ld of %s is %lld for %d columns", name, (long long)ld, cols);
    ACSC_CHECK_ARG(aligned(p, dtype_size(static_cast<acsc_dtype>(dt))), ACSC_EALIGN, "%s not aligned to its elements",
                   name);
    return ACSC_OK;
}

// A kept pre-activation: one of z and q.
inline int check_kept(const void *z, int64_t ldz, const q8_tensor *q, int64_t rows, int cols, int dt)
{
    ACSC_CHECK_ARG(rows == 0 || (z != nullptr) != (q != nullptr), ACSC_EINVAL, "exactly one of the tensor and its checkpoint is needed");
    if (z)
        return check_mat(z, true, ldz, cols, dt, "z");
    return q ? check_q8(q, rows, cols) : ACSC_OK;
}

inline int check_ws(const void *ws, size_t have, size_t need)
{
    if (need == 0)
        return ACSC_OK;
    ACSC_CHECK_ARG(ws, ACSC_EINVAL, "null workspace");
    ACSC_CHECK_ARG(aligned(ws, 256), ACSC_EALIGN, "workspace not 256-byte aligned");
    ACSC_CHECK_ARG(have >= need, ACSC_ENOSPC, "workspace of %zu bytes, %zu needed", have, need);
    return ACSC_OK;
}

// The largest launch of tiles: a grid has under 2^32 threads along x.
inline int check_tiles(const Plan &p)
{
    if (p.few)
        return ACSC_OK;
    const int64_t tiles = static_cast<int64_t>(p.tm) * p.tn, threads = 64 * waves(p.rows, p.tile);
    ACSC_CHECK_ARG(tiles * threads < (1ll << 32) && (p.whole + (tiles - p.whole) * p.splits) * threads < (1ll << 32),
                   ACSC_EINVAL, "product too large: %lld tiles of %d x %d", (long long)tiles, p.rows, p.tile);
    return ACSC_OK;
}

}  // namespace acsc
