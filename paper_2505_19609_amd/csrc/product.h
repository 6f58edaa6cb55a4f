// Products of two bf16 matrices in tiles, for the kernels of loss.hip and linear.hip: operands in LDS, the loop over the steps of a workgroup's tiles.
//
// A workgroup is 4 wavefronts, one per SIMD, and forms tiles of 64 NA x 64 NB (256 x 256, less where there are few rows): each wavefront 2 NA x 2 NB results of
// v_mfma_f32_16x16x32_bf16, so that an operand fragment read from LDS feeds several products.  Steps of 64 along the contraction lie in two LDS
// buffers (of 64 KB for 256 x 256), filled by loads that write LDS directly.  The chip's power decides the clock under such products: 16 x 16 x 32 needs less of it than 32 x 32 x 16, which moves
// each accumulator twice as often, and two products in a row on one accumulator less than by turns.
#pragma once

#include "tiles.h"

namespace {

constexpr int kTile = 256;       // rows and columns of a result tile
constexpr int kStep = 64;        // of the contraction
constexpr int kGrid = 256;       // workgroups: one per compute unit (tiles of 256 x 256 take as much LDS as allows no second one)

// Where an operand's step lies and how much of its matrix is behind that address.
struct Source {
    const unsigned char *at;
    int64_t left;
    uint32_t pitch;       // bytes between rows
    int64_t step;         // bytes from one step to the next
    __device__ __forceinline__ i32x4 words() const
    {
        const int64_t n = left < 0 ? 0 : left > 0x7fffffff ? 0x7fffffff : left;
        return rsrc_words(at, (uint32_t)n);
    }
    __device__ __forceinline__ void next() { at += step; left -= step; }
};

// A tile's operand in LDS: two halves, each of what the wavefronts read in a half of their blocks (of every 32 NB rows or columns
// the first or the second 16 NB; NB = 4: 16 KB a half).  A load's 64 pieces of 16 bytes lie one behind the other, so the arrangement is made
// on the global side: a lane fetches the piece that belongs where it writes.
//   ROWS  32 NB rows x 64 of the contraction (128 bytes a row): piece c of row r lies at c ^ (r / 2 & 7), so 16 rows' pieces of
//         one c, which are read together, are 16 different slots of the 256 bytes that the banks span.
//   COLS  64 of the contraction x 128 columns (256 bytes a row): piece c of row r lies at c ^ 2 (r & 3 | r / 2 & 4), so the 8 rows x 32 bytes
//         that a transposing read takes together are 16 different slots too.  NB = 1: x 32 columns (64 bytes a row), piece c at c ^ 2 (r / 8 & 1).
template <bool COLS, int NB>
struct Operand {
    static_assert(NB == 4 || NB == 1 || !COLS, "");
    static constexpr int kRowBytes = 64 * NB;   // (COLS) of a half
    static constexpr int kHalfBytes = 4096 * NB;
    int load[2];     // byte offsets of this lane's pieces in the tile's matrix: of even and odd instructions (COLS: of the first and the last two)
    int read[4];     // LDS offsets of its fragments: ROWS by half step (two), COLS by block of 16 columns

    // `part_rows` (ROWS): rows of the matrix from those of the first two wavefronts to those of the others
    __device__ __forceinline__ void init(int lane, int wave, int part, uint32_t pitch, int part_rows = 32 * NB)
    {
        const int s = lane & 15, g = lane >> 4;
        if (!COLS) {
#pragma unroll
            for (int o = 0; o < 2; ++o)
                load[o] = ((wave >> 1) * part_rows + (wave & 1) * 8 * NB + (lane >> 3)) * (int)pitch + (((lane & 7) ^ (4 * odd(o, wave) + (lane >> 4))) << 4);
#pragma unroll
            for (int k = 0; k < 2; ++k) read[k] = (part * 16 * NB + s) * 128 + (((4 * k + g) ^ (s >> 1)) << 4);
        } else {
#pragma unroll
            for (int o = 0; o < 2; ++o) {
                const int piece = NB == 4 ? s ^ (g + 4 * o) << 1 : (lane & 3) ^ (lane >> 5) << 1, row = NB == 4 ? g : lane >> 2;
                load[o] = (wave * 16 + row) * (int)pitch + (piece >> (NB == 4 ? 3 : 1)) * (64 * NB) + (piece & (2 * NB - 1)) * 16;
            }
#pragma unroll
            for (int t = 0; t < 4; ++t)
                read[t] = (8 * g + (s >> 2)) * kRowBytes + (((2 * NB * part + 2 * t + ((s & 3) >> 1)) ^ (NB == 4 ? (s >> 2) + 4 * (g & 1) : g & 1) << 1) << 4) + 8 * (s & 1);
        }
    }
    // This lane's offsets of a step.  `tail`: elements of the contraction that are left, where rows may end inside the
    // step (ROWS): what is behind them reads as zero.
    __device__ __forceinline__ void offsets(int lane, int wave, int tail, int off[2]) const
    {
#pragma unroll
        for (int o = 0; o < 2; ++o) {
            off[o] = load[o];
            if (!COLS && ((lane & 7) ^ (4 * odd(o, wave) + (lane >> 4))) * 8 >= tail) off[o] = (int)0x80000000;   // (past every descriptor's end)
        }
    }
    // whether an instruction fills an odd group of 8 rows: every second one of a wavefront does, or, where it has only one, every second wavefront's
    static __device__ __forceinline__ int odd(int o, int wave) { return NB == 1 ? wave & 1 : o; }
    // NB instructions of each wavefront fill a half.  `half_rows` (ROWS): rows of the matrix from the first half's to the second's
    __device__ __forceinline__ static void fetch(i32x4 words, const int off[2], uint32_t pitch, uint32_t lds, int wave, int half, int q, int half_rows = 16 * NB)
    {
        dma_b128(words, lds + half * kHalfBytes + (wave * NB + q) * 1024, off[COLS ? q >> 1 : q & 1],
                 COLS ? half * (32 * NB) + (int)(q * 4 * pitch) : (int)((half * half_rows + q * 8) * pitch));
    }
    // fragment b (16 rows or columns, 0..3) of a half and half step k: 8 consecutive elements of the contraction
    __device__ __forceinline__ bf16x8 get(const unsigned char *t, int half, int b, int k) const
    {
        if (!COLS) return *(const bf16x8 *)(t + read[k] + half * kHalfBytes + b * 2048);
        typedef s16x4 __attribute__((address_space(3))) * lds_ptr_t;
        const unsigned char *p = t + read[b] + half * kHalfBytes + k * (32 * kRowBytes);
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr_t)p);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr_t)(p + 4 * kRowBytes));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};

// A result that lies in an accumulator register.  (Read as ordinary values, all 256 were copied to vector registers at the end of the loop,
// and what was there before went to scratch memory.)
__device__ __forceinline__ float result(float f)
{
    float r;
    asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(r) : "a"(f));
    return r;
}

// Lane g of the four of a result column has rows 4 g .. 4 g + 3 of two blocks of 16.  In bf16, it gets rows 8 (g / 2) .. + 7 of the block g % 2.
__device__ __forceinline__ uint4 eight_of(const float *first, const float *second)
{
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    const u32x2 a = __builtin_amdgcn_permlane16_swap(pack_bf16(first[0], first[1]), pack_bf16(second[0], second[1]), false, false);
    const u32x2 b = __builtin_amdgcn_permlane16_swap(pack_bf16(first[2], first[3]), pack_bf16(second[2], second[3]), false, false);
    return make_uint4(a[0], b[0], a[1], b[1]);
}
// `x`, of which the compiler does not know that it is the same everywhere.  (What a seldom taken branch works out of it is worked out there then, and
// not ahead of them all.)
__device__ __forceinline__ int here(int x)
{
    asm volatile("" : "+v"(x));
    return x;
}
__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// Forms the tiles `begin`, `begin` + `stride`, .. below `end`: `lds` holds two buffers of kProductBytes<NA, NB>.
//   open(tile, a, b, steps, a_tail, b_tail)  where its operands' steps lie, how many there are (none: the tile has only an end), and, of an operand whose rows may
//                                            end inside a step (A_TAIL, B_TAIL), how many elements of the contraction
//   tile_begin(tile)                         before its products; returns the same number of steps
//   tile_end(acc)                            with its results: acc[x][y][v] is row 32 NA (wave & 1) + 16 x + 4 g + v and column 32 NB (wave >> 1) + 16 y + n of
//                                            the tile, g = lane / 16, n = lane % 16
template <int NA, int NB> constexpr int kProductBytes = 8192 * (NA + NB);
// `a_half_rows`: see Operand::fetch.
template <bool A_COLS, bool B_COLS, int NA, int NB, bool A_TAIL, bool B_TAIL, class Open, class Begin, class End>
__device__ __forceinline__ void product_tiles(unsigned char *lds, const Operand<A_COLS, NA> &A, const Operand<B_COLS, NB> &B, uint32_t a_pitch, uint32_t b_pitch, int begin, int end,
                                              int stride, Open open, Begin tile_begin, End tile_end, int a_half_rows = 16 * NA)
{
    constexpr int kOperandBytes = 8192 * NA, kBufferBytes = kProductBytes<NA, NB>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t lds0 = lds_addr(lds);

    // The steps of this workgroup's tiles are one sequence, and the loads run ahead in it across the end of a tile.
    struct Cursor {
        int tile, left, a_tail, b_tail, parity;
        Source a, b;
    };
    struct Fetch {   // what the loads of a step need
        i32x4 a, b;
        int a_off[2], b_off[2];
        uint32_t lds;
    };
    auto take = [&](Cursor &c) {   // the next step; behind the last one the loads read nothing
        while (c.left == 0 && c.tile < end) {
            open(c.tile, c.a, c.b, c.left, c.a_tail, c.b_tail);
            c.tile += stride;
        }
        if (c.left == 0) c.a.left = c.b.left = 0;
        Fetch f;
        f.a = c.a.words();
        f.b = c.b.words();
        A.offsets(lane, wave, A_TAIL ? c.a_tail : kStep, f.a_off);
        B.offsets(lane, wave, B_TAIL ? c.b_tail : kStep, f.b_off);
        f.lds = lds0 + c.parity * kBufferBytes;
        c.a.next();
        c.b.next();
        c.a_tail -= kStep;
        c.b_tail -= kStep;
        c.left -= c.left > 0;
        c.parity ^= 1;
        return f;
    };
    auto load_a = [&](const Fetch &f, int half, int q) { A.fetch(f.a, f.a_off, a_pitch, f.lds, wave, half, q, a_half_rows); };
    auto load_b = [&](const Fetch &f, int half, int q) { B.fetch(f.b, f.b_off, b_pitch, f.lds + kOperandBytes, wave, half, q); };

    // A step in two halves, of 64 products with NB = 4.  What a half of the blocks needs is read half a step before its first product, so its place
    // in LDS is free early, and its loads have a step until they are waited for:
    //   half  products        reads                       loads (of the step after next)
    //   1     A0 B0, A0 B1    B1, A1                      A0 B0
    //   2     A1 B0, A1 B1    A0, B0 of the next step     B1 A1
    // Each half ends with a barrier: what was read in it may be overwritten, and what the next one reads is there (a step's loads, 16 with NB = 4, are younger).
    bf16x8 a0[NA][2], a1[NA][2], b0[NB][2], b1[NB][2];   // [block of 16][half step]
    f32x4 acc[2 * NA][2 * NB];
    auto half_end = [&]() {
        SB();
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(2 * (NA + NB)) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        SB();
    };
    Cursor cursor = {begin, 0, 0, 0, 0, {}, {}};
#pragma unroll
    for (int step = 0; step < 2; ++step) {
        const Fetch f = take(cursor);
#pragma unroll
        for (int q = 0; q < NA; ++q) {
            load_a(f, 0, q);
            if (q < NB) load_b(f, 0, q);
        }
#pragma unroll
        for (int q = 0; q < NA; ++q) {
            if (q < NB) load_b(f, 1, q);
            load_a(f, 1, q);
        }
    }
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(3 * (NA + NB)) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    auto read_a = [&](const unsigned char *t, int half, bf16x8 to[NA][2], int i) { to[i % NA][i / NA] = A.get(t, half, i % NA, i / NA); };
    auto read_b = [&](const unsigned char *t, int half, bf16x8 to[NB][2], int i) { to[i % NB][i / NB] = B.get(t + kOperandBytes, half, i % NB, i / NB); };
#pragma unroll
    for (int j = 0; j < 2 * NA; ++j) {
        read_a(lds, 0, a0, j);
        if (j < 2 * NB) read_b(lds, 0, b0, j);
    }
    half_end();

    int at = 0;   // LDS offset of the step under way
    for (int i = begin; i < end; i += stride) {
        const int steps = tile_begin(i);
#pragma unroll
        for (int x = 0; x < 2 * NA; ++x)
#pragma unroll
            for (int y = 0; y < 2 * NB; ++y)
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[x][y][v] = 0.0f;
        for (int step = 0; step < steps; ++step) {
            const unsigned char *t = lds + at, *next = lds + (at ^ kBufferBytes);
            const Fetch f = take(cursor);
            if constexpr (NB == 4) {
                // Product j of a quarter: blocks j / 8 and j / 2 % 4, half step j % 2 (two products in a row on one accumulator need less power:
                // 1.7 % of the time against j / 16 for the half step); between pairs of them at most one read or load, i = j / 2.
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    const int k = j & 1, x = j >> 3 & 3, y = j >> 1 & 3, i = j >> 1;
                    acc[x][y] = mfma16(a0[x][k], b0[y][k], acc[x][y]);
                    SB();
                    if (j & 1) continue;
                    if (i < 8) b1[i >> 1][i & 1] = B.get(t + kOperandBytes, 1, i >> 1, i & 1);
                    else if (i & 1) load_b(f, 0, (i - 8) >> 1);
                    else load_a(f, 0, (i - 8) >> 1);
                    SB();
                }
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    const int k = j & 1, x = j >> 3 & 3, y = j >> 1 & 3, i = j >> 1;
                    acc[x][4 + y] = mfma16(a0[x][k], b1[y][k], acc[x][4 + y]);
                    SB();
                    if (j & 1) continue;
                    if (i < 8) a1[i >> 1][i & 1] = A.get(t, 1, i >> 1, i & 1);
                    SB();
                }
                half_end();
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    const int k = j & 1, x = j >> 3 & 3, y = j >> 1 & 3, i = j >> 1;
                    acc[4 + x][y] = mfma16(a1[x][k], b0[y][k], acc[4 + x][y]);
                    SB();
                    if (j & 1) continue;
                    if (i < 8) a0[i >> 1][i & 1] = A.get(next, 0, i >> 1, i & 1);
                    else if (i & 1) load_a(f, 1, (i - 8) >> 1);
                    else load_b(f, 1, (i - 8) >> 1);
                    SB();
                }
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    const int k = j & 1, x = j >> 3 & 3, y = j >> 1 & 3, i = j >> 1;
                    acc[4 + x][4 + y] = mfma16(a1[x][k], b1[y][k], acc[4 + x][4 + y]);
                    SB();
                    if (j & 1) continue;
                    if (i < 8) b0[i >> 1][i & 1] = B.get(next + kOperandBytes, 0, i >> 1, i & 1);
                    SB();
                }
                half_end();
            } else {   // (fewer products: memory is what is waited for, so the loads go first)
#pragma unroll
                for (int i = 0; i < NA; ++i) load_a(f, 0, i);
#pragma unroll
                for (int i = 0; i < NB; ++i) load_b(f, 0, i);
#pragma unroll
                for (int i = 0; i < 2 * NB; ++i) read_b(t, 1, b1, i);
#pragma unroll
                for (int i = 0; i < 2 * NA; ++i) read_a(t, 1, a1, i);
#pragma unroll
                for (int j = 0; j < 4 * NA * NB; ++j) {   // block of 16 rows of B, of A, half step
                    const int y = j / (2 * NA), x = j / 2 % NA, k = j & 1;
                    acc[x][y] = mfma16(a0[x][k], y < NB ? b0[y][k] : b1[y - NB][k], acc[x][y]);
                }
                half_end();
#pragma unroll
                for (int i = 0; i < NB; ++i) load_b(f, 1, i);
#pragma unroll
                for (int i = 0; i < NA; ++i) load_a(f, 1, i);
                bf16x8 b2[NB][2];   // (the first products of this half still need b0)
#pragma unroll
                for (int i = 0; i < 2 * NB; ++i) read_b(next, 0, b2, i);
#pragma unroll
                for (int i = 0; i < 2 * NA; ++i) read_a(next, 0, a0, i);
#pragma unroll
                for (int j = 0; j < 4 * NA * NB; ++j) {
                    const int y = j / (2 * NA), x = j / 2 % NA, k = j & 1;
                    acc[NA + x][y] = mfma16(a1[x][k], y < NB ? b0[y][k] : b1[y - NB][k], acc[NA + x][y]);
                }
#pragma unroll
                for (int i = 0; i < 2 * NB; ++i) b0[i / 2][i & 1] = b2[i / 2][i & 1];
                half_end();
            }
            at ^= kBufferBytes;
        }

        // (the compiler does not see that what follows reads results of the matrix pipe: the distance it would keep)
        asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
        tile_end(acc);
    }
    wait_vmem();   // (no load to LDS outlives the workgroup)
}


}  // namespace
