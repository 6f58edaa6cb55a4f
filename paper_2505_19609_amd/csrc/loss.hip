// Softmax cross entropy of packed rows times a vocabulary's weight, with its gradients (include/skrull_loss.h).
//
// Rows that have a target are gathered first (X: as many rows as there are, then zeros to a whole tile, hidden values
// padded with zeros to whole steps), so rows without one cost nothing and odd strides and alignments stay out of the products.
// How many there are only the device knows: every kernel reads it and works out its own tiles.
//
// Four products of the same shape, all on one tile kernel:
//   logits   z^T = W X^T           the forward keeps, per row and strip of 128 words, the largest logit and the sum of exponentials;
//            and again             the backward writes dz = d (exp(z - lse) - [word = target]) in bf16, a piece of the vocabulary at a time
//   dX       dz W                  fp32, added up over the pieces (and over parts of the vocabulary where there are few tiles)
//   dW^T     X^T dz                a piece's rows of dW are complete after one product
// What bounds them is the matrix pipe: 2 T V H operations each, against 2 (T + V) H bytes; with few rows reading W (37 rows, 896 hidden, 32,003 words, 57 MB:
// forward 23 us of which the product takes 13, backward 60 with W in the caches; 26 and 70 from memory).
//
// A workgroup is 4 wavefronts, one per SIMD, and forms a tile of 256 x 256 (x 64 or 128 where there are few rows): each wavefront 128 x 128, 8 x 8 results of
// v_mfma_f32_16x16x32_bf16 in 256 accumulator registers, so that an operand fragment read from LDS feeds eight products.  Steps of 64 along
// the contraction lie in two LDS buffers of 64 KB, filled by loads that write LDS directly.
// The chip's power decides the clock under such products, and with it what an instruction is worth: with normally distributed operands in registers and
// nothing else, 16 x 16 x 32 runs at 2,010 TFLOP/s, 32 x 32 x 16 (which moves each accumulator twice as often) at 1,705.  Here it is 1,340 to 1,400 (13,312 rows, 3,584
// hidden, 131,072 words: forward 9.0 ms, backward 28.2; torch's plain products of this size run at 1,440 to 1,520 on the same chip), whether the steps' barriers and
// waits are there or not: without them the matrix pipe is busier and the clock lower.
#include <math.h>

#include "ops.h"
#include "skrull_loss.h"
#include "tiles.h"

namespace {

constexpr int kTile = 256;       // rows and columns of a result tile
constexpr int kStep = 64;        // of the contraction
constexpr int kGrid = 256;       // workgroups: one per compute unit, each as much LDS as allows no second one
constexpr int64_t kPieceBytes = (int64_t)2 << 30;  // of dz at most, but for one tile of words of all rows: 640 bytes a row, more than that from 3.4 million rows on
// Rows of dz and of the gathered x are this much longer where their length is a multiple of 4 KB: the 256 rows of a tile would lie in few of the L2's sets.
constexpr int kPitchPad = 64;
constexpr int kMaxPieceWords = 1 << 20;            // (32-bit offsets within a tile of dz)
// With so few rows or fewer the backward has each of them twice, the second time with what rounding dz to bf16 leaves: dx and dw have no error but their own
// type's.  It costs little where W is what the products wait for (64 rows, 3,584 hidden, 128,000 words: backward 731 us and not 655; 37, 896, 32,003: 70 and 61).  (Where many
// rows add up, dz's roundings cost as much as the result's own: 2.4e-3 of a gradient's norm against 1.7e-3.  A single row's are all or nothing.)
constexpr int kTwice = kTile / 2;
// The second time begins at a multiple of 32: both together are a whole number of steps of dW (20 rows, 3,584 hidden, 60,000 words: dX and dW 189 us, 222 with
// multiples of 64).
constexpr int kTimes = kStep / 2;
__host__ __device__ inline int times_of(int64_t rows) { return (int)((rows + kTimes - 1) / kTimes * kTimes); }
// Where it begins, given the rows of dz and those that have a target; 0 if there is none.
__device__ __forceinline__ int second_of(const int32_t *n_rows) { return n_rows[0] > n_rows[1] ? n_rows[0] / 2 : 0; }
// Exponentials are exp2((z - shift) log2 e), the difference first: as z log2 e - shift log2 e, one instruction less, the second product's rounding is an error
// of 2^-24 of the logits in the exponent, which from 10^9 on left sums of 0 and infinity.  (0 to 0.7 % of the time.)
constexpr float kLog2e = 1.44269504088896340736f;

// What is taken off logits whose largest one this is: nothing where there is no word at all, or an infinite logit, so that a sum is 0 or infinite
// and not NaN.
__device__ __forceinline__ float shift_of(float most) { return fabsf(most) < INFINITY ? most : 0.0f; }
// What a sum of exponentials is multiplied by where its largest logit is `most` and that of all sums put together `all`: 1 at most.  (A sum of no words has nothing
// taken off; relative to logits of -100 its factor would be e^100 without the limit, relative to -89 and below infinite, and infinity times its zero no number.)
__device__ __forceinline__ float scale_of(float most, float all) { return fast_exp2(fminf((shift_of(most) - shift_of(all)) * kLog2e, 0.0f)); }

enum Kind { kForward, kAgain, kDx, kDw };

struct LossArgs {
    const uint16_t *x;       // gathered rows [.., xp], Hp of them used
    const uint16_t *w;       // [V, H]
    uint16_t *dz;            // [.., pitch of the pieces]
    const int32_t *n_rows;   // rows of dz, of them rows that have a target (and once more, second_of)
    const int32_t *target;   // of the gathered rows
    const float *lse, *d;    // of the gathered rows (kAgain)
    float *z_target;         // of the gathered rows (kForward)
    float2 *strips;          // [strips][Tp] (kForward)
    float *slabs;            // [splits][rows][Hp] (kDx)
    uint16_t *dw;            // [V, H] (kDw)
    int64_t Tp, dz_room;
    int32_t V, H, Hp, xp;    // xp: elements between rows of x
    int32_t piece;           // of the vocabulary, backward
};

// How many parts the vocabulary of a piece is cut into for dX, so that all compute units have a tile: the partial sums are slabs
// of their own, added up at the end in order.
__host__ __device__ inline int dx_splits(int tiles, int steps)
{
    const int s = kGrid / tiles;
    return s < 1 ? 1 : s > steps ? steps : s;
}

__host__ __device__ inline int row_tiles_of(int64_t rows) { return rows > 0 ? (int)((rows + kTile - 1) / kTile) : 1; }

// The pieces that the backward takes the vocabulary in: as few as the room for dz (in elements) allows for the rows there are, of equal
// size, or of one that gives dW fewer rounds of tiles on all compute units together.
struct Piece {
    int tiles, pitch;   // tiles of 256 words of a piece (the last one may have fewer); elements between rows of dz
    int most_pieces;    // with these rows or fewer
    __host__ __device__ Piece(int row_tiles, int V, int H, int64_t room)
    {
        const int words = (V + kTile - 1) / kTile, h_tiles = (H + kTile - 1) / kTile;
        int64_t most = (room / ((int64_t)row_tiles * kTile) - kPitchPad) / kTile;
        most = most < 1 ? 1 : most > kMaxPieceWords / kTile ? kMaxPieceWords / kTile : most;
        const int count = (int)((words + most - 1) / most);
        tiles = (words + count - 1) / count;
        most_pieces = count;
        int whole = kGrid;   // tiles that make whole rounds
        for (int h = h_tiles; whole > 1 && h % 2 == 0; h /= 2) whole /= 2;
        if (count > 1 && most >= whole) {
            const int other = (int)(most / whole * whole);
            if ((words + other - 1) / other <= most_pieces && rounds(words, other, h_tiles) < rounds(words, tiles, h_tiles)) tiles = other;
        }
        pitch = tiles * kTile + (tiles % 8 == 0 ? kPitchPad : 0);
    }
    __host__ __device__ static int rounds(int words, int tiles, int h_tiles)
    {
        const int rest = words % tiles;
        return words / tiles * ((tiles * h_tiles + kGrid - 1) / kGrid) + (rest * h_tiles + kGrid - 1) / kGrid;
    }
};

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
//         that a transposing read takes together are 16 different slots too.
template <bool COLS, int NB>
struct Operand {
    static_assert(NB == 4 || !COLS, "");
    static constexpr int kHalfBytes = 4096 * NB;
    int load[2];     // byte offsets of this lane's pieces in the tile's matrix: of even and odd instructions (COLS: of the first and the last two)
    int read[4];     // LDS offsets of its fragments: ROWS by half step (two), COLS by block of 16 columns

    __device__ __forceinline__ void init(int lane, int wave, int part, uint32_t pitch)
    {
        const int s = lane & 15, g = lane >> 4;
        if (!COLS) {
#pragma unroll
            for (int o = 0; o < 2; ++o)
                load[o] = ((wave >> 1) * 32 * NB + (wave & 1) * 8 * NB + (lane >> 3)) * (int)pitch + (((lane & 7) ^ (4 * odd(o, wave) + (lane >> 4))) << 4);
#pragma unroll
            for (int k = 0; k < 2; ++k) read[k] = (part * 16 * NB + s) * 128 + (((4 * k + g) ^ (s >> 1)) << 4);
        } else {
#pragma unroll
            for (int o = 0; o < 2; ++o) {
                const int piece = s ^ (g + 4 * o) << 1;
                load[o] = (wave * 16 + g) * (int)pitch + (piece >> 3) * 256 + (piece & 7) * 16;
            }
#pragma unroll
            for (int t = 0; t < 4; ++t)
                read[t] = (8 * g + (s >> 2)) * 256 + (((8 * part + 2 * t + ((s & 3) >> 1)) ^ ((s >> 2) + 4 * (g & 1)) << 1) << 4) + 8 * (s & 1);
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
    // NB instructions of each wavefront fill a half.
    __device__ __forceinline__ static void fetch(i32x4 words, const int off[2], uint32_t pitch, uint32_t lds, int wave, int half, int q)
    {
        dma_b128(words, lds + half * kHalfBytes + (wave * NB + q) * 1024, off[COLS ? q >> 1 : q & 1],
                 COLS ? half * 128 + (int)(q * 4 * pitch) : (int)((half * 16 * NB + q * 8) * pitch));
    }
    // fragment b (16 rows or columns, 0..3) of a half and half step k: 8 consecutive elements of the contraction
    __device__ __forceinline__ bf16x8 get(const unsigned char *t, int half, int b, int k) const
    {
        if (!COLS) return *(const bf16x8 *)(t + read[k] + half * kHalfBytes + b * 2048);
        typedef s16x4 __attribute__((address_space(3))) * lds_ptr_t;
        const unsigned char *p = t + read[b] + half * kHalfBytes + k * 8192;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr_t)p);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr_t)(p + 1024));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
};

// The tiles of a product and their operands.
template <Kind K, int NA, int NB>
struct Product {
    static constexpr int kRows = 64 * NB;   // columns of a tile: rows of x, but for kDw
    static constexpr int kWords = 64 * NA;  // its rows: words, or (256) hidden values
    int mt, nt, splits, steps, total;   // tiles of M and N; parts of the contraction, steps of a part
    int v0, zp, all_steps;              // first word of the piece; elements between rows of dz; kDx: steps of all parts

    __device__ __forceinline__ void init(const LossArgs &p, int n_rows)
    {
        const int row_tiles = max(1, (n_rows + kRows - 1) / kRows), h_tiles = (p.H + kTile - 1) / kTile, words = (p.V + kTile - 1) / kTile;
        splits = 1;
        v0 = zp = all_steps = 0;
        int piece_tiles = (p.V + kWords - 1) / kWords;
        if (K != kForward) {
            const Piece piece(row_tiles_of(n_rows), p.V, p.H, p.dz_room);
            zp = piece.pitch;
            v0 = p.piece * piece.tiles * kTile;
            piece_tiles = max(0, min(piece.tiles, words - p.piece * piece.tiles)) * (kTile / kWords);   // (no tile: there are fewer pieces than launches)
            splits = K == kDx ? dx_splits(h_tiles * row_tiles, piece.tiles * (kTile / kStep)) : 1;
        }
        if (K == kForward || K == kAgain) {
            mt = piece_tiles;
            nt = row_tiles;
            steps = p.Hp / kStep;
        } else if (K == kDx) {
            mt = piece_tiles ? h_tiles : 0;
            nt = row_tiles;
            all_steps = piece_tiles * (kTile / kStep);
            steps = (all_steps + splits - 1) / splits;
        } else {
            mt = h_tiles;
            nt = piece_tiles;
            steps = max(1, (n_rows + kStep - 1) / kStep);
        }
        total = mt * nt * splits;
        for (int *f : {&mt, &nt, &splits, &steps, &total, &v0, &zp, &all_steps}) *f = __builtin_amdgcn_readfirstlane(*f);   // (quotients come from vector instructions)
    }
    // Tiles in the order of work: blocks of 8 tiles of M, through all of N.  Neighbours in it run at the same time on one die, 8 x 4 tiles
    // that share their operands in its L2.
    __device__ __forceinline__ void locate(int i, int &m, int &n, int &s) const
    {
        s = i / (mt * nt);
        i -= s * (mt * nt);
        const int block = i / (8 * nt), r = i - block * (8 * nt), width = min(8, mt - block * 8);
        n = r / width;
        m = block * 8 + r - n * width;
        for (int *f : {&m, &n, &s}) *f = __builtin_amdgcn_readfirstlane(*f);
    }
    // steps of part s (the last one may have fewer, or none)
    __device__ __forceinline__ int steps_of(int s) const
    {
        return K == kDx ? max(0, min(steps, all_steps - s * steps)) : steps;
    }
    __device__ __forceinline__ void sources(const LossArgs &p, int m, int n, int s, Source &a, Source &b) const
    {
        const int64_t H2 = (int64_t)p.H * 2, xp2 = (int64_t)p.xp * 2, zp2 = (int64_t)zp * 2;
        if (K == kForward || K == kAgain) {
            const int64_t v = v0 + (int64_t)m * kWords;
            a = Source{(const unsigned char *)p.w + v * H2, min((int64_t)kWords, p.V - v) * H2, (uint32_t)H2, kStep * 2};
            b = Source{(const unsigned char *)p.x + (int64_t)n * kRows * xp2, kRows * xp2, (uint32_t)xp2, kStep * 2};
        } else if (K == kDx) {
            const int64_t k0 = (int64_t)s * steps * kStep;
            a = Source{(const unsigned char *)p.w + (v0 + k0) * H2 + m * kTile * 2, (p.V - v0 - k0) * H2 - m * kTile * 2, (uint32_t)H2, kStep * H2};
            b = Source{(const unsigned char *)p.dz + (int64_t)n * kRows * zp2 + k0 * 2, kRows * zp2 - k0 * 2, (uint32_t)zp2, kStep * 2};
        } else {
            const int64_t rows = (int64_t)steps * kStep;
            a = Source{(const unsigned char *)p.x + m * kTile * 2, rows * xp2 - m * kTile * 2, (uint32_t)xp2, kStep * xp2};
            b = Source{(const unsigned char *)p.dz + (int64_t)n * kTile * 2, rows * zp2 - (int64_t)n * kTile * 2, (uint32_t)zp2, kStep * zp2};
        }
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

// The tile is 64 NA x 64 NB: 256 x 256, x 128 or 64 with few rows, 64 x 64 with few words too (the logits).
template <Kind K, int NA, int NB>
__global__ __launch_bounds__(256, 1) void loss_product_kernel(const LossArgs p)
{
    static_assert(NA == 4 || (NA == 1 && NB == 1 && (K == kForward || K == kAgain)), "");
    constexpr bool A_COLS = K == kDx || K == kDw, B_COLS = K == kDw;
    // (what the results of a tile need of its rows comes by loads to LDS too, in two places by turns: a load to registers would be waited for
    // together with all that are under way)
    constexpr int kRows = 64 * NB, kOperandBytes = 8192 * NA, kBufferBytes = kOperandBytes + 8192 * NB, kStrip = 32 * NA;
    constexpr int kRowBytes = K == kForward ? kRows * 4 : K == kAgain ? 3 * kRows * 4 : 0;
    __shared__ __align__(1024) unsigned char lds[2 * kBufferBytes + 2 * kRowBytes];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave & 1, wn = wave >> 1;
    const int n = lane & 15, g = lane >> 4;
    const int n_rows = __builtin_amdgcn_readfirstlane(p.n_rows[K == kForward || K == kAgain]);
    Product<K, NA, NB> work;
    work.init(p, n_rows);

    const uint32_t a_pitch = (uint32_t)(K == kDw ? p.xp : p.H) * 2, b_pitch = (uint32_t)(K == kDx || K == kDw ? work.zp : p.xp) * 2;
    Operand<A_COLS, NA> A;
    Operand<B_COLS, NB> B;
    A.init(lane, wave, wm, a_pitch);
    B.init(lane, wave, wn, b_pitch);
    const uint32_t lds0 = lds_addr(lds);

    const int die = blockIdx.x & 7, per_die = (work.total + 7) / 8, stride = gridDim.x >> 3;
    const int begin = die * per_die + (blockIdx.x >> 3), end = min(work.total, (die + 1) * per_die);

    // The steps of this workgroup's tiles are one sequence, and the loads run ahead in it across the end of a tile.
    struct Cursor {
        int tile, left, tail, parity;
        Source a, b;
    };
    struct Fetch {   // what the loads of a step need
        i32x4 a, b;
        int a_off[2], b_off[2];
        uint32_t lds;
    };
    auto take = [&](Cursor &c) {   // the next step; behind the last one the loads read nothing
        while (c.left == 0 && c.tile < end) {
            int m, nn, s;
            work.locate(c.tile, m, nn, s);
            c.left = work.steps_of(s);
            work.sources(p, m, nn, s, c.a, c.b);
            c.tail = K == kForward || K == kAgain ? p.H : 0x7fffffff;   // elements of the contraction
            c.tile += stride;
        }
        if (c.left == 0) c.a.left = c.b.left = 0;
        Fetch f;
        f.a = c.a.words();
        f.b = c.b.words();
        A.offsets(lane, wave, c.tail, f.a_off);
        B.offsets(lane, wave, kStep, f.b_off);
        f.lds = lds0 + c.parity * kBufferBytes;
        c.a.next();
        c.b.next();
        c.tail -= kStep;
        c.left -= c.left > 0;
        c.parity ^= 1;
        return f;
    };
    auto load_a = [&](const Fetch &f, int half, int q) { A.fetch(f.a, f.a_off, a_pitch, f.lds, wave, half, q); };
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
    Cursor cursor = {begin, 0, 0, 0, {}, {}};
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

    int at = 0, row_at = 2 * kBufferBytes;   // LDS offsets of the step under way and of the tile's row data
    for (int i = begin; i < end; i += stride) {
        int m, nn, s;
        work.locate(i, m, nn, s);
        const int steps = work.steps_of(s);
        if (K == kForward || K == kAgain) {
            const int row0 = nn * kRows + wave * 64;   // (older than a step's loads: there when the first one ends)
            if (wave < NB) {
                dma_b32(rsrc_words(p.target + row0, 256), lds0 + row_at + wave * 256, lane * 4, 0);
                if (K == kAgain) {
                    dma_b32(rsrc_words(p.lse + row0, 256), lds0 + row_at + 4 * kRows + wave * 256, lane * 4, 0);
                    dma_b32(rsrc_words(p.d + row0, 256), lds0 + row_at + 8 * kRows + wave * 256, lane * 4, 0);
                }
            }
        }
        const int *row_targets = (const int *)(lds + row_at);
        const float *row_lse = (const float *)(lds + row_at + 4 * kRows), *row_d = (const float *)(lds + row_at + 8 * kRows);
        row_at ^= (2 * kBufferBytes) ^ (2 * kBufferBytes + kRowBytes);
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
        // acc[x][y][v] is row 32 NA wm + 16 x + 4 g + v and column 32 NB wn + 16 y + n of the tile
        if (K == kForward) {
            const int strip = m * 2 + wm;
            const int words = p.V - strip * kStrip - 4 * g;   // of the strip, from this lane's first one on
            const bool whole = (m * 2 + wm + 1) * kStrip <= p.V;
            float most[2 * NB], sum[2 * NB];   // of this lane's words; the four lanes of a row are put together at the end
#pragma unroll
            for (int y = 0; y < 2 * NB; ++y) {
                const int in_tile = wn * 32 * NB + y * 16 + n, row = nn * kRows + in_tile;
                SB();
                float z[8 * NA];
#pragma unroll
                for (int j = 0; j < 8 * NA; ++j) z[j] = result(acc[j >> 2][y][j & 3]);
                if (!whole) {
                    const int left = here(words);
#pragma unroll
                    for (int j = 0; j < 8 * NA; ++j)
                        if (16 * (j >> 2) + (j & 3) >= left) z[j] = -INFINITY;
                }
                float a[2] = {z[0], z[1]}, b[8];
#pragma unroll
                for (int j = 2; j < 8 * NA; ++j) a[j & 1] = fmaxf(a[j & 1], z[j]);
                most[y] = fmaxf(a[0], a[1]);
                const float shift = shift_of(most[y]);
                const int t = row_targets[in_tile] - strip * kStrip;
                if (__any(t >= 0 && t < kStrip)) {
                    const int mine = (t >> 2 & 3) == g && t >= 0 && t < kStrip ? (t >> 4) * 4 + (t & 3) : -1;
                    float found = z[0];
#pragma unroll
                    for (int j = 1; j < 8 * NA; ++j) found = j == mine ? z[j] : found;
                    if (mine >= 0) p.z_target[row] = found;
                }
#pragma unroll
                for (int i = 0; i < NA; ++i) {   // (eight at a time: an exponential's result is not ready for the next instruction)
                    float e[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) e[j] = fast_exp2((z[8 * i + j] - shift) * kLog2e);
                    SB();
#pragma unroll
                    for (int j = 0; j < 8; ++j) b[j] = i == 0 ? e[j] : b[j] + e[j];
                }
                sum[y] = ((b[0] + b[1]) + (b[2] + b[3])) + ((b[4] + b[5]) + (b[6] + b[7]));
                asm volatile("" : "+v"(most[y]), "+v"(sum[y]));   // (formed here, not for all y at the end, with all logits in registers)
            }
            SB();
#pragma unroll
            for (int y = 0; y < 2 * NB; ++y) {
                const float all = fmaxf(fmaxf(most[y], __shfl_xor(most[y], 16)), fmaxf(__shfl_xor(most[y], 32), __shfl_xor(most[y], 48)));
                sum[y] *= scale_of(most[y], all);
                most[y] = all;
            }
#pragma unroll
            for (int y = 0; y < 2 * NB; ++y) sum[y] += __shfl_xor(sum[y], 16);
#pragma unroll
            for (int y = 0; y < 2 * NB; ++y) sum[y] += __shfl_xor(sum[y], 32);
            float2 *out = p.strips + (int64_t)strip * p.Tp + nn * kRows + wn * 32 * NB + n;
#pragma unroll
            for (int y = 0; y < 2 * NB; ++y)
                if (g == (y & 3)) out[y * 16] = make_float2(most[y], sum[y]);
        } else if (K == kAgain) {
            const int word0 = m * work.kWords + wm * kStrip;   // of the piece
            const int words = p.V - work.v0 - word0 - 4 * g;
            const bool whole = work.v0 + word0 + kStrip <= p.V;
            const int second = second_of(p.n_rows), rows = second ? second : max(1, (n_rows + kStep - 1) / kStep) * kStep;   // rows: that dW's product reads, each time
            const bool twice = second > 0;
            const bool filled = (nn + 1) * kRows > n_rows;   // (with rows that fill the last tile)
#pragma unroll
            for (int y = 0; y < 2 * NB; ++y) {
                const int in_tile = wn * 32 * NB + y * 16 + n, row = nn * kRows + in_tile;
                const float lse = row_lse[in_tile], d = row_d[in_tile];
                const int t = row_targets[in_tile] - work.v0 - word0;
                const bool hit = __any(t >= 0 && t < kStrip);
                const int mine = (t >> 2 & 3) == g && t >= 0 && t < kStrip ? (t >> 4) * 4 + (t & 3) : -1;
                uint16_t *out = p.dz + (int64_t)row * work.zp + word0 + 16 * (g & 1) + 8 * (g >> 1);
#pragma unroll
                for (int x = 0; x < 2 * NA; x += 2) {
                    SB();
                    float e[8];   // of two blocks
#pragma unroll
                    for (int v = 0; v < 8; ++v) e[v] = fast_exp2((result(acc[x + (v >> 2)][y][v & 3]) - lse) * kLog2e);
                    if (hit) {
                        const int at = here(mine) - 4 * x;
#pragma unroll
                        for (int v = 0; v < 8; ++v)
                            if (v == at) e[v] -= 1.0f;
                    }
#pragma unroll
                    for (int v = 0; v < 8; ++v) e[v] *= d;
                    if (!whole) {
                        const int left = here(words) - 16 * x;
#pragma unroll
                        for (int v = 0; v < 8; ++v)
                            if (16 * (v >> 2) + (v & 3) >= left) e[v] = 0.0f;
                    }
                    if (filled) {   // (their logits are 0 times w, which may hold infinities: no number, and nor is its product with a d of 0)
                        const bool none = here(row) >= n_rows;
#pragma unroll
                        for (int v = 0; v < 8; ++v) e[v] = none ? 0.0f : e[v];
                    }
                    const uint4 u = eight_of(e, e + 4);
                    if (row < rows) *(uint4 *)(out + x * 16) = u;
                    if (twice) {
#pragma unroll
                        for (int v = 0; v < 8; ++v) e[v] -= __builtin_bit_cast(float, pack_bf16(0.0f, e[v]) & 0xffff0000u);
                        const uint4 rest = eight_of(e, e + 4);
                        if (row < rows) *(uint4 *)(out + (int64_t)rows * work.zp + x * 16) = rest;
                    }
                }
            }
        } else if (K == kDx) {
            float *out = p.slabs + ((int64_t)(s * work.nt + nn) * kRows + wn * 32 * NB) * p.Hp + m * kTile + wm * 128;   // (the same for all lanes)
            const int cols = p.H - m * kTile - wm * 128;
            const int valid = p.n_rows[1], again = second_of(p.n_rows);
#pragma unroll
            for (int y = 0; y < 2 * NB; ++y) {
                float *row = out + y * 16 * p.Hp;
                const int r = nn * kRows + wn * 32 * NB + y * 16 + n;
                const bool stored = r < valid || (again && r >= again && r - again < valid);   // (not the zeros behind either time)
                const uint32_t mine = n * p.Hp + 4 * g;
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    SB();
                    if (stored && x * 16 + 4 * g < cols) {   // (a whole number of fours)
                        float4 *to = (float4 *)(row + x * 16 + mine);
                        float4 f = make_float4(result(acc[x][y][0]), result(acc[x][y][1]), result(acc[x][y][2]), result(acc[x][y][3]));
                        if (p.piece > 0) {
                            const float4 old = *to;
                            f.x += old.x; f.y += old.y; f.z += old.z; f.w += old.w;
                        }
                        *to = f;
                    }
                }
            }
        } else {
            const int col0 = m * kTile + wm * 128 + 16 * (g & 1) + 8 * (g >> 1);
#pragma unroll
            for (int y = 0; y < 2 * NB; ++y) {
                const int word = work.v0 + nn * kTile + wn * 128 + y * 16 + n;
                uint16_t *out = p.dw + (int64_t)word * p.H + col0;
#pragma unroll
                for (int x = 0; x < 8; x += 2) {
                    SB();
                    float e[8];
#pragma unroll
                    for (int v = 0; v < 8; ++v) e[v] = result(acc[x + (v >> 2)][y][v & 3]);
                    const uint4 u = eight_of(e, e + 4);
                    if (word < p.V && col0 + x * 16 < p.H) *(uint4 *)(out + x * 16) = u;
                }
            }
        }
    }
    wait_vmem();   // (no load to LDS outlives the workgroup)
}

// X: the rows that have a target, in order, then zeros to a whole tile; and what else the products need of them.  A workgroup has `each` rows; how many
// of those before them have a target it counts itself, 8 bytes a row that lie in the L2 (16,384 rows, 896 hidden: rows
// and copies 12 us; with one workgroup for the rows and a launch of its own for the copies 36).
struct GatherArgs {
    const uint16_t *x;
    int64_t x_stride;
    const int64_t *target;   // [T]
    const float *lse, *d;    // [T], backward
    int64_t T;
    int32_t V, H, Hp, xp, each, wide;
    int32_t *n_rows, *slot, *row, *target_of;  // [2], see LossArgs; [T] gathered row or -1; [Tp] its row; [Tp] its target
    uint16_t *out;           // [Tp][xp]
    float *lse_of, *d_of;    // [Tp], backward
    float *loss, *lse_out;   // [T], forward: zeros where there is no target
    float *z_target;         // [Tp], forward: NaN until the product finds the target's word
};
constexpr int kGatherWaves = 16;
template <bool BACKWARD>
__global__ __launch_bounds__(64 * kGatherWaves) void loss_gather_kernel(const GatherArgs a)
{
    __shared__ int counts[2][kGatherWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t first = (int64_t)blockIdx.x * a.each, end = min(a.T, first + a.each);
    int before = 0, n = 0;
#pragma unroll 8
    for (int64_t t = threadIdx.x; t < a.T; t += 64 * kGatherWaves) {
        const int has = a.target[t] >= 0;
        n += has;
        before += t < first ? has : 0;
    }
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) {
        n += __shfl_xor(n, m);
        before += __shfl_xor(before, m);
    }
    if (lane == 0) {
        counts[0][wave] = before;
        counts[1][wave] = n;
    }
    __syncthreads();
    int at = 0;
    n = 0;
#pragma unroll
    for (int k = 0; k < kGatherWaves; ++k) {
        at += counts[0][k];
        n += counts[1][k];
    }
    const bool twice = BACKWARD && n > 0 && n <= kTwice;
    const int again = times_of(n);   // the second time
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        a.n_rows[0] = twice ? 2 * again : n;
        a.n_rows[1] = n;
    }

    for (int64_t t0 = first; t0 < end; t0 += 64) {
        const int64_t t = t0 + lane, target = t < end ? a.target[t] : -1;
        const uint64_t has = __ballot(target >= 0);
        if (wave == 0 && t < end) {
            const int s = at + __popcll(has & (((uint64_t)1 << lane) - 1));
            a.slot[t] = target >= 0 ? s : -1;
            if (target >= 0) {
                const bool outside = target >= a.V;
                a.row[s] = (int32_t)t;
                a.target_of[s] = outside ? -1 : (int32_t)target;
                if (BACKWARD) {
                    a.lse_of[s] = a.lse[t];
                    a.d_of[s] = outside ? NAN : a.d[t];
                } else {
                    a.z_target[s] = NAN;
                }
            } else if (!BACKWARD) {
                a.loss[t] = 0.0f;
                a.lse_out[t] = 0.0f;
            }
        }
        for (int i = wave; i < 64; i += kGatherWaves) {
            if (!(has >> i & 1)) continue;
            const uint16_t *in = a.x + (t0 + i) * a.x_stride;
            uint16_t *to = a.out + (int64_t)(at + __popcll(has & (((uint64_t)1 << i) - 1))) * a.xp;
#pragma unroll 4
            for (int c = lane * 8; c < a.Hp; c += 64 * 8) {
                uint4 v = make_uint4(0, 0, 0, 0);
                if (c < a.H) {
                    if (a.wide) {
                        v = *(const uint4 *)(in + c);
                    } else {
                        uint16_t e[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) e[k] = in[c + k];
                        v = make_uint4(e[0] | (uint32_t)e[1] << 16, e[2] | (uint32_t)e[3] << 16, e[4] | (uint32_t)e[5] << 16, e[6] | (uint32_t)e[7] << 16);
                    }
                }
                *(uint4 *)(to + c) = v;
                if (twice) *(uint4 *)(to + (int64_t)again * a.xp + c) = v;
            }
        }
        at += __popcll(has);
    }
    const int padded = row_tiles_of(n) * kTile;
    for (int r = n + blockIdx.x + wave * gridDim.x; r < padded; r += gridDim.x * kGatherWaves) {   // rows that fill the last tile: no gradient, no word
        if (lane == 0) {
            a.target_of[r] = -1;
            if (BACKWARD) { a.lse_of[r] = 0.0f; a.d_of[r] = 0.0f; }
        }
        if (twice && r >= again && r < again + n) continue;
        for (int c = lane * 8; c < a.Hp; c += 64 * 8) *(uint4 *)(a.out + (int64_t)r * a.xp + c) = make_uint4(0, 0, 0, 0);
    }
}

// lse and loss from the strips: 16 rows to a workgroup, 64 lanes of a row share its strips.
constexpr int kSumRows = 16;
__global__ __launch_bounds__(1024) void loss_sums_kernel(const float2 *strips, int n_strips, int64_t Tp, const int32_t *n_rows, const int32_t *row,
                                                         const float *z_target, float *loss, float *lse)
{
    __shared__ float2 part[64][kSumRows + 1];
    const int i = threadIdx.x % kSumRows, share = threadIdx.x / kSumRows, r0 = blockIdx.x * kSumRows, n = *n_rows;
    if (r0 >= n) return;
    // largest logit and the sum of exponentials relative to it
    auto add = [&](float2 &a, float2 b) {
        const float m = fmaxf(a.x, b.x);
        a.y = a.y * scale_of(a.x, m) + b.y * scale_of(b.x, m);
        a.x = m;
    };
    float2 sum = make_float2(-INFINITY, 0.0f);
    for (int k = share; k < n_strips; k += 64 * 8) {   // (eight loads at a time, to the last one)
        float2 part_of[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) part_of[j] = strips[min(k + 64 * j, n_strips - 1) * Tp + r0 + i];   // (within the padded rows)
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (k + 64 * j < n_strips) add(sum, part_of[j]);
    }
    part[share][i] = sum;
    __syncthreads();
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;   // a wavefront to a row
    sum = part[lane][wave];
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) add(sum, make_float2(__shfl_xor(sum.x, m), __shfl_xor(sum.y, m)));
    const int r = r0 + wave;
    if (lane == 0 && r < n) {
        const float l = shift_of(sum.x) + logf(sum.y);
        const int t = row[r];
        lse[t] = l;
        loss[t] = l - z_target[r];
    }
}

// dx of every row: the parts' sums, or zeros.  A thread has 4 columns, SHARES threads share their parts: 4 where there are 32 parts or more, whose loads
// would be many waits one after another (37 rows, 896 hidden, 63 parts: 5.5 us, 10.0 by one thread; 2,000 rows, 8 parts: 22.6, 16.4 by one).
template <int SHARES>
__device__ __forceinline__ void sum_parts(const float *slabs, int64_t slab, int splits, int64_t rest, const int32_t *slot, uint16_t *dx, int64_t T, int H, int Hp)
{
    constexpr int kThreads = 256 / SHARES;
    __shared__ float4 part[SHARES][SHARES > 1 ? kThreads : 1];
    const int share = threadIdx.x / kThreads, blocks = (H / 4 + kThreads - 1) / kThreads;
    for (int64_t i = blockIdx.x; i < T * blocks; i += gridDim.x) {
        const int64_t t = i / blocks;
        const int c = ((int)(i - t * blocks) * kThreads + threadIdx.x % kThreads) * 4, s = slot[t];
        float4 f = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        auto add = [&](float4 u) { f.x += u.x; f.y += u.y; f.z += u.z; f.w += u.w; };
        if (s >= 0 && c < H) {
            const float *from = slabs + (int64_t)s * Hp + c + share * slab;
            for (int times = rest ? 2 : 1; times > 0; --times, from = slabs + (int64_t)s * Hp + c + share * slab + rest) {
                int k = share;
                for (; k + 7 * SHARES < splits; k += 8 * SHARES, from += 8 * SHARES * slab) {
                    float4 u[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) u[j] = *(const float4 *)(from + j * SHARES * slab);
#pragma unroll
                    for (int j = 0; j < 8; ++j) add(u[j]);
                }
                for (; k < splits; k += SHARES, from += SHARES * slab) add(*(const float4 *)from);
            }
        }
        if constexpr (SHARES > 1) {
            __syncthreads();   // (what the row before left is read)
            part[share][threadIdx.x % kThreads] = f;
            __syncthreads();
            if (share == 0)
#pragma unroll
                for (int k = 1; k < SHARES; ++k) add(part[k][threadIdx.x]);
        }
        if (share == 0 && c < H) *(uint2 *)(dx + t * H + c) = make_uint2(pack_bf16(f.x, f.y), pack_bf16(f.z, f.w));
    }
}
__global__ __launch_bounds__(256) void loss_dx_kernel(const float *slabs, const int32_t *n_rows, const int32_t *slot, uint16_t *dx, int64_t T, int V, int H, int Hp,
                                                      int64_t dz_room, int tile_rows)
{
    const int n = n_rows[0], tiles = max(1, (n + tile_rows - 1) / tile_rows);
    const int splits = dx_splits(tiles * ((H + kTile - 1) / kTile), Piece(row_tiles_of(n), V, H, dz_room).tiles * (kTile / kStep));
    const int64_t slab = (int64_t)tiles * tile_rows * Hp, rest = (int64_t)second_of(n_rows) * Hp;   // rest: to the products of what was left of dz
    if (splits >= 32) sum_parts<4>(slabs, slab, splits, rest, slot, dx, T, H, Hp);
    else sum_parts<1>(slabs, slab, splits, rest, slot, dx, T, H, Hp);
}

// How many rows of x the products with the vocabulary's words take at a time: 64 where tiles of 256 leave compute units without one, as many as there
// are where they are up to 128, so that memory is what is waited for.  In us, of the forward:
//   rows, hidden, words     64 at a time  128  256
//   37, 896, 32,003                   25         38
//   64, 3,584, 128,000               172        210
//   128, 896, 32,003                  24   29    37
//   128, 3,584, 128,000              236  181   215
//   192, 896, 150,000                 90         89
//   256, 896, 32,003                  34         36
//   512, 896, 150,000                210        141
// And 64 words, four workgroups to a compute unit, where that leaves half of the compute units without a tile still (forward's product and backward's, us:
// 100 rows, 896 hidden, 4,000 words 9.7 and 10.0, with 256 words 14.6 and 16.0; 300, 1,200, 5,000 14.8 and 14.8, 18.8 and 19.4; 37, 896, 32,003 13.0 and 14.2, 15.1 and
// 17.0; but 128, 896, 32,003 17.1 and 19.3, 15.0 and 19.0).
struct Tile { int words, rows; };
Tile logits_tile(int64_t rows, int vocab)
{
    const int64_t tiles = (rows + 63) / 64 * ((vocab + kTile - 1) / kTile);
    if (2 * tiles <= kGrid) return {64, 64};
    if (rows <= 64 || tiles <= 2 * kGrid) return {kTile, 64};
    return {kTile, rows <= 128 ? 128 : kTile};
}
// The workspace, from sizes alone.
struct Layout {
    int64_t Tp, Hp, xp, dz_room, pieces;
    int64_t n_rows, slot, row, target, lse, d, z_target, x, strips, dz, slabs, bytes;
    Layout(const skrull_loss_t &p, bool backward)
    {
        const int64_t row_tiles = row_tiles_of(p.rows);
        Tp = row_tiles * kTile;
        Hp = (p.hidden + kStep - 1) / kStep * kStep;
        xp = Hp * 2 % 4096 == 0 ? Hp + kPitchPad : Hp;
        const int64_t words = ((int64_t)p.vocab + kTile - 1) / kTile * kTile;
        bytes = dz_room = pieces = 0;
        auto take = [&](int64_t n) { const int64_t at = bytes; bytes += (n + 255) & ~(int64_t)255; return at; };
        n_rows = take(8);
        slot = take(p.rows * 4);
        row = take(Tp * 4);
        target = take(Tp * 4);
        x = take(Tp * xp * 2);
        lse = d = z_target = strips = dz = slabs = 0;
        if (backward) {
            lse = take(Tp * 4);
            d = take(Tp * 4);
            // (one tile of the vocabulary at least, however many rows there are)
            const int64_t all = Tp * ((words < kMaxPieceWords ? words : kMaxPieceWords) + kPitchPad), least = Tp * (kTile + kPitchPad);
            dz_room = all < kPieceBytes / 2 ? all : kPieceBytes / 2 > least ? kPieceBytes / 2 : least;
            pieces = Piece((int)row_tiles, p.vocab, p.hidden, dz_room).most_pieces;
            dz = take(dz_room * 2);
            // (parts of the vocabulary are made only where there are fewer tiles than compute units)
            const int64_t h_tiles = (p.hidden + kTile - 1) / kTile, parted = kGrid / h_tiles * kTile;
            slabs = take((Tp > parted ? Tp : parted) * Hp * 4);
        } else {
            z_target = take(Tp * 4);
            strips = take(words / (logits_tile(p.rows, p.vocab).words / 2) * Tp * 8);
        }
    }
};

int check(const skrull_loss_t *p)
{
    if (!p) return refuse("loss: null pointer");
    if (p->rows < 0 || p->rows > 1 << 24) return refuse("loss: %lld rows", (long long)p->rows);
    if (p->hidden < 8 || p->hidden > 65536 || p->hidden % 8 != 0) return refuse("loss: hidden %d is not a multiple of 8 from 8 to 65536", p->hidden);
    if (p->vocab < 1 || p->vocab > 1 << 22) return refuse("loss: vocab %d", p->vocab);
    if (p->x_stride < p->hidden || p->x_stride > (int64_t)1 << 32) return refuse("loss: x_stride %lld", (long long)p->x_stride);
    return SKRULL_OK;
}

// The same of dX's product, whose parts fill the compute units: 64 where even so the tiles are few (256 rows, 896 hidden, 32,003 words: backward 91 us,
// 96 with 256; 600, 128, 4,000: 48 and 55; but 512, 896, 150,000: 562 and 480).  Up to kTwice rows may be there twice.
int dx_tile_rows_of(int64_t rows, int hidden)
{
    if (rows <= kTwice) rows = 2 * times_of(rows);
    if (rows <= 128) return rows <= 64 ? 64 : 128;
    return (rows + 63) / 64 * ((hidden + kTile - 1) / kTile) <= 16 ? 64 : kTile;
}
template <Kind K>
hipError_t launch(Tile tile, const LossArgs &a, hipStream_t st)
{
    if constexpr (K == kForward || K == kAgain)
        if (tile.words == 64) {
            loss_product_kernel<K, 1, 1><<<4 * kGrid, 256, 0, st>>>(a);   // (as many fit the compute units)
            return hipGetLastError();
        }
    if (tile.rows == 64) loss_product_kernel<K, 4, 1><<<kGrid, 256, 0, st>>>(a);
    else if (tile.rows == 128) loss_product_kernel<K, 4, 2><<<kGrid, 256, 0, st>>>(a);
    else loss_product_kernel<K, 4, 4><<<kGrid, 256, 0, st>>>(a);
    return hipGetLastError();
}

// The first kernel of either direction.
template <bool BACKWARD>
hipError_t gather(const skrull_loss_t &p, const Layout &l, unsigned char *ws, const void *x, const int64_t *target, const float *lse, const float *d,
                  float *loss, float *lse_out, hipStream_t st)
{
    GatherArgs a = {};
    a.x = (const uint16_t *)x; a.x_stride = p.x_stride; a.target = target; a.lse = lse; a.d = d; a.T = p.rows; a.V = p.vocab;
    a.H = p.hidden; a.Hp = (int32_t)l.Hp; a.xp = (int32_t)l.xp; a.wide = aligned_to(x, 16) && p.x_stride % 8 == 0;
    a.each = (int32_t)((p.rows + 511) / 512 < 4 ? 4 : (p.rows + 511) / 512);
    a.n_rows = (int32_t *)(ws + l.n_rows); a.slot = (int32_t *)(ws + l.slot); a.row = (int32_t *)(ws + l.row); a.target_of = (int32_t *)(ws + l.target);
    a.out = (uint16_t *)(ws + l.x); a.lse_of = (float *)(ws + l.lse); a.d_of = (float *)(ws + l.d); a.loss = loss; a.lse_out = lse_out; a.z_target = (float *)(ws + l.z_target);
    const int64_t blocks = (p.rows + a.each - 1) / a.each;   // (16 and more: a few rows' workgroups write the zeros behind them too)
    loss_gather_kernel<BACKWARD><<<(int)(blocks < 16 ? 16 : blocks), 64 * kGatherWaves, 0, st>>>(a);
    return hipGetLastError();
}

LossArgs args_of(const skrull_loss_t &p, const Layout &l, unsigned char *ws, const void *w)
{
    LossArgs a = {};
    a.x = (const uint16_t *)(ws + l.x); a.w = (const uint16_t *)w;
    a.n_rows = (const int32_t *)(ws + l.n_rows); a.target = (const int32_t *)(ws + l.target);
    a.Tp = l.Tp; a.V = p.vocab; a.H = p.hidden; a.Hp = (int32_t)l.Hp; a.xp = (int32_t)l.xp;
    return a;
}

}  // namespace

extern "C" {

int64_t skrull_loss_workspace(const skrull_loss_t *p, int backward)
{
    return check(p) == SKRULL_OK ? Layout(*p, backward != 0).bytes : 0;
}

int skrull_loss_fwd(const skrull_loss_t *p, const void *x, const void *w, const int64_t *target, float *loss, float *lse,
                    void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (int rc = check(p)) return rc;
    if (p->rows == 0) return SKRULL_OK;
    if (!x || !aligned_to(x, 2) || !w || !aligned_to(w, 16) || !target || !aligned_to(target, 8) || !loss || !aligned_to(loss, 4) || !lse ||
        !aligned_to(lse, 4) || !workspace || !aligned_to(workspace, 16))
        return refuse("loss: null or misaligned pointer");
    const Layout l(*p, false);
    if ((int64_t)workspace_bytes < l.bytes) return refuse("loss: workspace below %lld bytes", (long long)l.bytes);
    int compute_units = 0;
    if (int rc = current_device(&compute_units)) return rc;
    unsigned char *ws = (unsigned char *)workspace;
    hipStream_t st = (hipStream_t)hip_stream;
    hipError_t e = gather<false>(*p, l, ws, x, target, nullptr, nullptr, loss, lse, st);
    if (e == hipSuccess) {
        LossArgs a = args_of(*p, l, ws, w);
        a.z_target = (float *)(ws + l.z_target);
        a.strips = (float2 *)(ws + l.strips);
        const Tile tile = logits_tile(p->rows, p->vocab);
        e = launch<kForward>(tile, a, st);
        if (e == hipSuccess) {
            loss_sums_kernel<<<(int)(l.Tp / kSumRows), 1024, 0, st>>>(a.strips, (p->vocab + tile.words - 1) / tile.words * 2, l.Tp, a.n_rows, (const int32_t *)(ws + l.row), a.z_target, loss, lse);
            e = hipGetLastError();
        }
    }
    return e == hipSuccess ? SKRULL_OK : launch_failed(e, "loss launch");
}

int skrull_loss_bwd(const skrull_loss_t *p, const void *x, const void *w, const int64_t *target, const float *lse, const float *d_loss,
                    void *dx, void *dw, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (int rc = check(p)) return rc;
    if (!dx && !dw) return SKRULL_OK;
    if (!w || !aligned_to(w, 16) || !aligned_to(dx, 16) || !aligned_to(dw, 16) || !workspace || !aligned_to(workspace, 16))
        return refuse("loss: null or misaligned pointer");
    if (p->rows > 0 && (!x || !aligned_to(x, 2) || !target || !aligned_to(target, 8) || !lse || !aligned_to(lse, 4) || !d_loss || !aligned_to(d_loss, 4)))
        return refuse("loss: null or misaligned pointer");
    const Layout l(*p, true);
    if ((int64_t)workspace_bytes < l.bytes) return refuse("loss: workspace below %lld bytes", (long long)l.bytes);
    const int64_t w_bytes = (int64_t)p->vocab * p->hidden * 2, dx_bytes = p->rows * p->hidden * 2;
    if ((dw && overlap(w, w_bytes, dw, w_bytes)) || (dx && overlap(w, w_bytes, dx, dx_bytes)) || (dx && dw && overlap(dw, w_bytes, dx, dx_bytes)))
        return refuse("loss: dx or dw overlaps w or the other");
    int compute_units = 0;
    if (int rc = current_device(&compute_units)) return rc;
    unsigned char *ws = (unsigned char *)workspace;
    hipStream_t st = (hipStream_t)hip_stream;
    hipError_t e = gather<true>(*p, l, ws, x, target, lse, d_loss, nullptr, nullptr, st);
    LossArgs a = args_of(*p, l, ws, w);
    a.lse = (const float *)(ws + l.lse);
    a.d = (const float *)(ws + l.d);
    a.dz = (uint16_t *)(ws + l.dz);
    a.slabs = (float *)(ws + l.slabs);
    a.dw = (uint16_t *)dw;
    a.dz_room = l.dz_room;
    const Tile tile = logits_tile(p->rows, p->vocab);
    const int dx_rows = dx_tile_rows_of(p->rows, p->hidden);
    for (int64_t i = 0; i < l.pieces && e == hipSuccess; ++i) {   // (there may be fewer pieces: the last launches find no tiles then)
        a.piece = (int32_t)i;
        e = launch<kAgain>(tile, a, st);
        if (e == hipSuccess && dx) {
            e = launch<kDx>(Tile{kTile, dx_rows}, a, st);
        }
        if (e == hipSuccess && dw) {
            loss_product_kernel<kDw, 4, 4><<<kGrid, 256, 0, st>>>(a);
            e = hipGetLastError();
        }
    }
    if (e == hipSuccess && dx && p->rows > 0) {
        const int64_t blocks = p->rows * ((p->hidden / 4 + 63) / 64);
        loss_dx_kernel<<<(int)(blocks < 4096 ? blocks : 4096), 256, 0, st>>>(a.slabs, a.n_rows, (const int32_t *)(ws + l.slot), (uint16_t *)dx, p->rows, p->vocab, p->hidden, (int)l.Hp, l.dz_room, dx_rows);
        e = hipGetLastError();
    }
    return e == hipSuccess ? SKRULL_OK : launch_failed(e, "loss launch");
}

}  // extern "C"
