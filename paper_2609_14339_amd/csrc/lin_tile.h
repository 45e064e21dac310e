// The tiled products of the linear layers, on v_mfma_f32_16x16x32_bf16 and
// v_mfma_f32_16x16x4_f32.
//
// A workgroup takes a TM x T tile of C in steps of 128 bytes along the sum (64
// bf16, 32 fp32): 256 x 256 (bf16 only) by eight waves of 64 rows and 128
// columns, 128 x 128 by four of 32 rows, and, for few rows, 64 x 128 by four of
// 16 and 32 x 128 by two, for few columns 128 x 64 by four of 32.
// Each step's tiles of A and B come straight from memory into LDS
// (global_load_lds_dwordx4); no register holds them on the way.  An operand
// stays in LDS as it is stored: lines of one index's step (row) or k-lines of
// 128 bytes of its own indices (col), their eight 16-byte chunks XOR-swizzled
// by the line.  Fragments are 16-byte reads of row operands; of col ones pairs
// of transposing 8-byte reads (bf16) or four 4-byte reads (fp32); so all three
// products of a layer run at the stored layouts.  The matrix instruction's
// first operand is B's side: a lane then holds four consecutive columns of a
// row.
//
// Half a step of fragments is read ahead.  While the first half of a step is
// multiplied the second is read, and A of two steps on leaves for the third of
// its stages; then the wave waits for what it sent of the next step, meets the
// others, sends B of two steps on into the stage just read, and multiplies the
// second half while the next step's first is read.  So the DMA, which bounds
// the kernel, is under way all the time: with two stages of both operands,
// all of it behind the meeting, 8192 x 28672 -> 8192 forward took 2850 us and
// 2720 so.  (Four waves of 128 x 128 keep 256 accumulators a lane, which the
// compiler moves between register files all the time; steps of half the length
// in rings of three to five stages read lines of 64 bytes and lose 8%.)
//
// Measured, TFLOP/s, forward / input gradient / weight gradient: bf16 8192 x
// 28672 -> 8192 1448 / 1385 / 1361, 8192 x 8192 -> 8192 1441 / 1385 / 1364,
// 16384 x 2048 -> 8192 1297 / 1336 / 1360; fp32 4096^3 147 / 144 / 137 of 157
// that the matrix cores have at 2.4 GHz.  What bounds it: at 8192 x 28672 ->
// 8192 the products alone, from registers, run at 2260 (the clock is near 1.7
// GHz by then), with their LDS reads at 1750, the DMA alone, two
// stages deep, at 1450.
#pragma once

#include "lin.h"

#include <atomic>
#include <type_traits>

namespace acsc {
namespace {

typedef __attribute__((__vector_size__(8 * sizeof(short)))) short bf16x8;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) unsigned char lds_byte;


// What lanes past the end of the sum read in its last step.
__device__ const uint4 g_zeros = {0, 0, 0, 0};

// As for the streaming passes: neither the 16-byte reads of 16 lines nor the
// transposed 8-byte reads of four lines conflict.
__device__ __forceinline__ int swz(int line) { return ((line >> 1) ^ line) & 7; }

// LDS DMA of 16 bytes a lane from base + off (bytes) to lds + 16 lane, or of 4
// bytes a lane from p to lds + 4 lane.  lds is wave-uniform and goes through
// M0, which needs a wait state after it is written; M0 is left as it was.
__device__ __forceinline__ void dma16(const char *base, uint32_t off, uint32_t lds)
{
    uint32_t saved;
    asm volatile("s_mov_b32 %0, m0\n\t"
                 "s_mov_b32 m0, %3\n\t"
                 "s_nop 0\n\t"
                 "global_load_lds_dwordx4 %1, %2\n\t"
                 "s_mov_b32 m0, %0"
                 : "=&s"(saved)
                 : "v"(off), "s"(base), "s"(lds)
                 : "memory");
}
__device__ __forceinline__ void dma16(const void *p, uint32_t lds)
{
    uint32_t saved;
    asm volatile("s_mov_b32 %0, m0\n\t"
                 "s_mov_b32 m0, %2\n\t"
                 "s_nop 0\n\t"
                 "global_load_lds_dwordx4 %1, off\n\t"
                 "s_mov_b32 m0, %0"
                 : "=&s"(saved)
                 : "v"(p), "s"(lds)
                 : "memory");
}
__device__ __forceinline__ void dma4(const void *p, uint32_t lds)
{
    uint32_t saved;
    asm volatile("s_mov_b32 %0, m0\n\t"
                 "s_mov_b32 m0, %2\n\t"
                 "s_nop 0\n\t"
                 "global_load_lds_dword %1, off\n\t"
                 "s_mov_b32 m0, %0"
                 : "=&s"(saved)
                 : "v"(p), "s"(lds)
                 : "memory");
}

// One operand's side of the DMA: N instructions a wave and step for the tile's
// T indices.  Instruction d of the T / 8 moves lines 8 d .. 8 d + 7: line l of a row operand is its
// index l, chunk c its c-th 16 bytes of k; line l of a col operand is k = l %
// BK of the l / BK-th 128 bytes of indices, chunk c 16 bytes of them.  Indices
// past the end are read as the last ones (their results are not stored); a col
// operand's last 16 bytes of a row may run on into the next row.
// GLU: the rows of a gated product's W, of which every 128 lines hold 64 of the
// gate and the 64 up ones that belong to them; a wave's lines are of one kind,
// i0 their first index.
template <typename E, bool COL, int T, int N, bool GLU = false>
struct Side {
    static_assert(!GLU || (!COL && (N == 4 || N == 8)), "a wave's lines lie in one block of 64");
    static constexpr int ES = sizeof(E), BK = 128 / ES, EC = 16 / ES;
    uint32_t off[N];       // bytes from the step's base
    const char *base;      // the tile's first index at the step's first k
    int64_t step;          // bytes from one step's base to the next

    __device__ __forceinline__ void init(const Operand &o, int64_t i0, int64_t ni, int k0, int wave)
    {
        const int lane = threadIdx.x & 63;
        const int64_t ld = o.ld * ES;
        base = static_cast<const char *>(o.p) + (COL ? k0 * ld + i0 * ES : i0 * ld + static_cast<int64_t>(k0) * ES);
        step = COL ? BK * ld : BK * ES;
        const int last = static_cast<int>(min<int64_t>(ni - i0, T)) - 1;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int d = wave * N + i, line = GLU ? (d * 8 + (lane >> 3)) & 63 : d * 8 + (lane >> 3), k = line % BK;
            const int c = (lane & 7) ^ swz(COL ? k : line);
            if (COL)
                off[i] = static_cast<uint32_t>(k * ld + min(line / BK * BK + c * EC, last & ~(EC - 1)) * ES);
            else
                off[i] = static_cast<uint32_t>(min(line, last) * ld + c * 16);
        }
    }
    // The sum's last step of `left` k, zeros past the end.  In chunks where a row
    // operand is readable, and zero, up to the next multiple of one, or a col
    // operand's indices are whole chunks (or readable up to there).
    __device__ __forceinline__ void chunks(int64_t s, int left, int wave, uint32_t lds) const
    {
        const int lane = threadIdx.x & 63;
        const char *from = base + s * step;
        asm volatile("" : "+v"(from));   // in vector registers here, so that the whole steps' stays in scalar ones
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int line = (wave * N + i) * 8 + (lane >> 3), k = COL ? line % BK : ((lane & 7) ^ swz(line)) * EC;
            dma16(k < left ? static_cast<const void *>(from + off[i]) : static_cast<const void *>(&g_zeros), lds + i * 1024);
        }
    }
    // Word by word otherwise: nothing is read past a row operand's k or the end
    // of a col operand.
    __device__ __forceinline__ void words(int64_t s, int left, int last, int64_t ld, int wave, uint32_t lds) const
    {
        constexpr int EW = 4 / ES;       // elements of a word
        const int lane = threadIdx.x & 63;
        const char *from = base + s * step;
        asm volatile("" : "+v"(from));
#pragma unroll 4
        for (int q = 0; q < 4 * N; ++q) {
            const int line = GLU ? (wave * N * 8 + q * 2 + (lane >> 5)) & 63 : wave * N * 8 + q * 2 + (lane >> 5), at = lane & 31;
            const int kl = line % BK, e = ((at >> 2) ^ swz(COL ? kl : line)) * EC + (at & 3) * EW;
            const int k = COL ? kl : e;
            const int64_t by = COL ? kl * ld + min(line / BK * BK + e, last & ~(EW - 1)) * ES : min(line, last) * ld + e * ES;
            dma4(k < left ? static_cast<const void *>(from + by) : static_cast<const void *>(&g_zeros), lds + q * 256);
        }
    }
};

// Fragment t of 16 indices, k half kh of a stage.  bf16: lane L holds index
// L % 16, k = 32 kh + 8 (L / 16) .. + 7.  fp32: index L % 16, k = 16 kh +
// 4 (L / 16) .. + 3, one for each of four instructions.
template <typename E, bool COL>
struct Frag;
template <bool COL>
struct Frag<uint16_t, COL> {
    typedef bf16x8 Value;
    uint32_t row[2];        // row: byte offset per k half
    uint32_t col[4][2];     // col: per 16 indices of a 64-wide block, k lines + 0 and + 4
    __device__ __forceinline__ void init(int t0)   // the wave's first fragment of its block
    {
        const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4;
        if (!COL) {
#pragma unroll
            for (int kh = 0; kh < 2; ++kh)
                row[kh] = l16 * 128 + 16 * ((kh * 4 + g) ^ swz(l16));
        } else {
            // ds_read_b64_tr_b16: result lane L, element e of each group of 16
            // lanes = element L % 4 of what lane 4 e + L / 4 read; lane 4 e + q
            // reads indices 4 q .. 4 q + 3 of k-line e.
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int line = g * 8 + (l16 >> 2) + 4 * h, x = ((t0 + t) & 3) * 16 + (l16 & 3) * 4;
                    col[t][h] = line * 128 + 16 * ((x >> 3) ^ swz(line)) + (x & 7) * 2;
                }
        }
    }
    __device__ __forceinline__ Value read(const unsigned char *op, int t, int kh) const
    {
        if (!COL)
            return *reinterpret_cast<const bf16x8 *>(op + row[kh] + t * 2048);
        const unsigned char *p = op + (t >> 2) * 8192 + kh * 4096;
        const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_s16x4 *>((lds_byte *)(p + col[t & 3][0])));
        const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_s16x4 *>((lds_byte *)(p + col[t & 3][1])));
        return bf16x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    }
    static __device__ __forceinline__ f32x4 multiply(const Value &b, const Value &a, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, a, c, 0, 0, 0);
    }
    static constexpr int kBlock = 64;   // indices of a col operand's 128 bytes
};
template <bool COL>
struct Frag<float, COL> {
    typedef f32x4 Value;
    uint32_t row[2];
    uint32_t col[2][4];     // per 16 indices of a 32-wide block, k
    __device__ __forceinline__ void init(int t0)
    {
        const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4;
        if (!COL) {
#pragma unroll
            for (int kh = 0; kh < 2; ++kh)
                row[kh] = l16 * 128 + 16 * ((kh * 4 + g) ^ swz(l16));
        } else {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int line = g * 4 + e, x = ((t0 + t) & 1) * 16 + l16;
                    col[t][e] = line * 128 + 16 * ((x >> 2) ^ swz(line)) + (x & 3) * 4;
                }
        }
    }
    __device__ __forceinline__ Value read(const unsigned char *op, int t, int kh) const
    {
        if (!COL)
            return *reinterpret_cast<const f32x4 *>(op + row[kh] + t * 2048);
        const unsigned char *p = op + (t >> 1) * 4096 + kh * 2048;
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            v[e] = *reinterpret_cast<const float *>(p + col[t & 1][e]);
        return v;
    }
    static __device__ __forceinline__ f32x4 multiply(const Value &b, const Value &a, f32x4 c)
    {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(b[e], a[e], c, 0, 0, 0);
        return c;
    }
    static constexpr int kBlock = 32;
};

// Stages of A: a third one where it fits beside the other workgroup (see the
// step below); B has two.
constexpr int a_stages(int TM) { return TM < 128 ? 2 : 3; }

template <typename E, int TM, int T, bool ACOL, bool BCOL, int KIND, typename TO>
__global__ __launch_bounds__(64 * waves(TM, T), TM == 64 ? 3 : 2) void lin_tile_kernel(Gemm g)
{
    extern __shared__ __align__(1024) unsigned char smem[];
    static_assert(!ACOL || TM >= 64, "a col operand A fills whole blocks");
    constexpr int kBK = 128 / sizeof(E);
    constexpr int WN = T < 128 ? 1 : T / 128;   // waves along the columns
    constexpr int FB = T < 128 ? T / 16 : 8;    // 16-column fragments of a wave
    constexpr int FA = fragments(TM);
    constexpr int OPA = TM * 128, OPB = T * 128;   // bytes of a step's A and B
    constexpr int AS = a_stages(TM);
    constexpr int B0 = AS * OPA;                // B's stages follow A's
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;

    // Workgroups go to the eight XCDs in turn; each XCD takes a run of tiles
    // of its own.  First the whole tiles, then the pieces of the others, a
    // piece of each in turn.
    uint32_t id = blockIdx.x, count = g.whole, first = 0;
    int split = -1;
    if (id >= count) {
        first = count;
        count = static_cast<uint32_t>(g.tm) * g.tn - first;
        split = static_cast<int>((id - first) / count);
        id = id - first - split * count;
    }
    {
        const uint32_t q = count / 8, r = count % 8, x = id % 8;
        id = x * q + min(x, r) + id / 8;
    }
    float *part = split < 0 ? nullptr : g.part + (static_cast<int64_t>(split) * count + id) * TM * T;
    int tile_m, tile_n;
    tile_at(g, first + id, tile_m, tile_n);
    const int64_t m0 = static_cast<int64_t>(tile_m) * TM;
    constexpr bool GLU = KIND == kGluForward;
    constexpr int TC = GLU ? T / 2 : T;         // columns of the output
    const int n0 = tile_n * TC;
    const int kbeg = split < 0 ? 0 : split * g.kchunk;
    const int kend = split < 0 ? g.K : kbeg + min(g.K - kbeg, g.kchunk);
    const int nsteps = (kend - kbeg - 1) / kBK + 1;   // kend - kbeg up to 2^31 - 1
    // steps of whole chunks: not a partial one, nor the sum's last where a col
    // operand's last chunk would run on past its end
    const bool ragged = (ACOL && g.words_a) || (BCOL && g.words_b);
    const int whole = (kend - kbeg) / kBK - (ragged && kend == g.K && g.K % kBK == 0);
    const int lasta = static_cast<int>(min<int64_t>(g.M - m0, TM)) - 1;

    // DMA instructions of a wave and step
    constexpr int NA = TM / 8 / waves(TM, T), NB = T / 8 / waves(TM, T);
    Side<E, ACOL, TM, NA> sa;
    Side<E, BCOL, T, NB, GLU> sb;
    sa.init(g.A, m0, g.M, kbeg, wave);
    int lastb = min(g.N - n0, T) - 1;
    if constexpr (GLU) {
        // this wave's lines; a block past the end reads the last row
        const int line = wave * NB * 8, i0 = min(n0 + line / 128 * 64, g.N - 1);
        const E *w = static_cast<const E *>(g.B.p) + (line & 64 ? g.N * g.B.ld : 0);
        lastb = min(g.N - i0, 64) - 1;
        sb.init(Operand{w, g.B.ld}, i0, i0 + lastb + 1, kbeg, wave);
    } else {
        sb.init(g.B, n0, g.N, kbeg, wave);
    }
    typedef Frag<E, ACOL> FragA;
    typedef Frag<E, BCOL> FragB;
    FragA fra;
    FragB frb;
    constexpr int BA = FragA::kBlock / 16;      // fragments of a col operand's block
    fra.init(wm * FA % BA);
    frb.init(0);
    const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_byte *)smem));

    constexpr int NR = (FB + FA - 1) / FA + 1;  // fragments read beside a row of products
    // instruction i of step s, which is whole, into stage `at`
    const auto issue_a = [&](int s, int at, int i) {
        dma16(sa.base + s * sa.step, sa.off[i], lds0 + at * OPA + (wave * NA + i) * 1024);
    };
    const auto issue_b = [&](int s, int i) {
        dma16(sb.base + s * sb.step, sb.off[i], lds0 + B0 + (s & 1) * OPB + (wave * NB + i) * 1024);
    };
    // all of any step, into A's stage `at` (A and B leave in turn)
    const auto any_a = [&](int s, int at) {
        if (s < whole) {
#pragma unroll
            for (int i = 0; i < NA; ++i)
                issue_a(s, at, i);
        } else if (s < nsteps) {
            const int left = kend - kbeg - s * kBK;
            const uint32_t to = lds0 + at * OPA + wave * NA * 1024;
            if (g.words_a)
                sa.words(s, left, lasta, g.A.ld * sizeof(E), wave, to);
            else
                sa.chunks(s, left, wave, to);
        }
    };
    const auto any_b = [&](int s) {
        if (s < whole) {
#pragma unroll
            for (int i = 0; i < NB; ++i)
                issue_b(s, i);
        } else if (s < nsteps) {
            const int left = kend - kbeg - s * kBK;
            const uint32_t to = lds0 + B0 + (s & 1) * OPB + wave * NB * 1024;
            if (g.words_b)
                sb.words(s, left, lastb, g.B.ld * sizeof(E), wave, to);
            else
                sb.chunks(s, left, wave, to);
        }
    };
    f32x4 acc[FA][8];
#pragma unroll
    for (int a = 0; a < FA; ++a)
#pragma unroll
        for (int j = 0; j < 8; ++j)
            acc[a][j] = f32x4{0, 0, 0, 0};
    // fragments of k half kh of a stage: FB of B's side, then FA of A's
    struct Frags {
        typename FragA::Value f[FB + FA];
    };
    const auto read = [&](Frags &f, int s, int at, int kh, int r) {
        if (r >= FB + FA)
            return;
        if (r < FB)
            f.f[r] = frb.read(smem + B0 + (s & 1) * OPB + wn * 16384, r, kh);
        else
            f.f[r] = fra.read(smem + at * OPA + (ACOL ? wm * FA / BA * (BA * 2048) : wm * FA * 2048), r - FB, kh);
    };
    // a row of products at a time, with what goes out beside them
    const auto multiply = [&](const Frags &f, int a) {
#pragma unroll
        for (int j = 0; j < FB; ++j)
            acc[a][j] = FragA::multiply(f.f[j], f.f[FB + a], acc[a][j]);
    };
    // this wave's DMA has landed, but for the newest `ahead`, and its LDS reads
    // are done; then everyone's
    const auto meet = [&](auto ahead) {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"i"(ahead.value) : "memory");
    };
    typedef std::integral_constant<int, 0> All;
    typedef std::integral_constant<int, AS == 3 ? NA : 0> ButA;
    Frags f0, f1;
    int at = 0;                                 // A's stage of the step at hand
    const auto step = [&](int s, auto inner) {   // inner: step s + 2 goes in chunks
        const int at1 = at + 1 == AS ? 0 : at + 1, at2 = at1 + 1 == AS ? 0 : at1 + 1;
#pragma unroll
        for (int a = 0; a < FA; ++a) {
            __builtin_amdgcn_sched_barrier(0);
            if (AS == 3)
#pragma unroll
                for (int i = 0; i < NA / FA; ++i)
                    if (inner)
                        issue_a(s + 2, at2, a * (NA / FA) + i);
#pragma unroll
            for (int r = 0; r < NR; ++r)
                read(f1, s, at, 1, a * NR + r);
            multiply(f0, a);
        }
        if (inner) {
            meet(ButA{});
        } else {
            meet(All{});
            any_a(s + 2, at2);
            any_b(s + 2);
        }
#pragma unroll
        for (int a = 0; a < FA; ++a) {
            __builtin_amdgcn_sched_barrier(0);
            if (AS == 2)
#pragma unroll
                for (int i = 0; i < NA / FA; ++i)
                    if (inner)
                        issue_a(s + 2, at2, a * (NA / FA) + i);
#pragma unroll
            for (int i = 0; i < NB / FA; ++i)
                if (inner)
                    issue_b(s + 2, a * (NB / FA) + i);
            // past the last step this reads another stage, unused
#pragma unroll
            for (int r = 0; r < NR; ++r)
                read(f0, s + 1, at1, 0, a * NR + r);
            multiply(f1, a);
        }
        at = at1;
    };

    for (int s = 0; s < 2; ++s) {
        any_a(s, s);
        any_b(s);
    }
    if (whole >= 2)
        meet(std::integral_constant<int, NA + NB>{});
    else
        meet(All{});
#pragma unroll
    for (int r = 0; r < FB + FA; ++r)
        read(f0, 0, 0, 0, r);
    int s = 0;
    for (; s + 2 < whole; ++s)
        step(s, std::true_type{});
    for (; s < nsteps; ++s)
        step(s, std::false_type{});
    meet(All{});
    if (tile_n == 0 && split <= 0)
        put_db<KIND>(g, m0, TM);
    if (part)
        part += wm * FA * 16 * T + wn * 128;
    constexpr int PUT = FA < 2 ? FA : 2;        // fragments' rows at a time
    char *own = reinterpret_cast<char *>(smem) + wave * PUT * 8192;
    float sg[8] = {}, su[8] = {};
#pragma unroll
    for (int a = 0; a < FA; a += PUT)
        put_tile<TO, KIND, PUT, WN>(g, reinterpret_cast<const f32x4(&)[PUT][8]>(acc[a]), own, m0 + (wm * FA + a) * 16,
                               n0 + wn * (GLU ? 64 : 128), min(g.N, n0 + TC), part ? part + a * 16 * T : nullptr, T,
                               wn, sg, su);
    if constexpr (KIND == kGluGate) {
        // the waves' column sums meet in LDS, in order: four lanes hold eight
        // columns of every fourth row each
        if (g.e.sums && !part) {
            constexpr int WM = waves(TM, T) / WN, WC = FB * 16;
            float *at = reinterpret_cast<float *>(smem);
            __syncthreads();
            const int lane = threadIdx.x & 63;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                sg[i] += __shfl_xor(sg[i], 16);
                su[i] += __shfl_xor(su[i], 16);
                sg[i] += __shfl_xor(sg[i], 32);
                su[i] += __shfl_xor(su[i], 32);
                if (lane * 8 < WC && lane < 16) {
                    at[(wm * 2 + 0) * T + wn * 128 + lane * 8 + i] = sg[i];
                    at[(wm * 2 + 1) * T + wn * 128 + lane * 8 + i] = su[i];
                }
            }
            __syncthreads();
            float *out = g.e.sums + static_cast<int64_t>(tile_m) * 2 * g.N;
            for (int c = threadIdx.x; c < 2 * T; c += blockDim.x) {
                float s = 0.f;
#pragma unroll
                for (int w = 0; w < WM; ++w)
                    s += at[w * 2 * T + c];
                const int half = c / T, n = n0 + c % T;
                if (n < g.N)
                    out[static_cast<int64_t>(half) * g.N + n] = s;
            }
        }
    }
}

template <typename E, int TM, int T, bool ACOL, bool BCOL, int KIND, typename TO>
int launch(const Gemm &g, hipStream_t st, const char *tag)
{
    constexpr size_t bytes = (a_stages(TM) * TM + 2 * T) * 128;
    // once a device: asked for on every call it costs the host more than the launch
    static std::atomic<uint64_t> allowed{0};
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess)
        return set_error(ACSC_EHIP, "cannot query the device");
    if (dev > 63 || !(allowed.load(std::memory_order_relaxed) >> dev & 1)) {
        if (int rc = allow_lds(lin_tile_kernel<E, TM, T, ACOL, BCOL, KIND, TO>, bytes))
            return rc;
        if (dev < 64)
            allowed.fetch_or(1ull << dev, std::memory_order_relaxed);
    }
    ACSC_LAUNCH(tag, (lin_tile_kernel<E, TM, T, ACOL, BCOL, KIND, TO>),
                dim3(g.whole + (g.tm * g.tn - g.whole) * g.splits), dim3(64 * waves(TM, T)), bytes, st, g);
    return check_launch(tag);
}

}  // namespace
}  // namespace acsc
