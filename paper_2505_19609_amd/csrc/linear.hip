// The product of packed rows and a weight with bias, activation, gate and residual, and its gradients (include/skrull_linear.h).
//
// Three products on the tile loop of product.h:
//   z^T  = W X^T     what follows it is done where a tile's results leave the accumulators
//   dX   = dZ W
//   dW^T = X^T dZ
// dz is formed once, by a kernel of its own (dy and z to dz, and the sums over rows for db), since both other products read it.  Without an activation it is dy itself.
//
// Two things have fewer bits than 32 on their way.  z is kept in bf16 from the forward to the backward: y is formed before that rounding, and in 32 bits z would be 763 MB more to
// write and to read again at 13,312 rows of 2 x 14,336, 0.3 ms of 6.8.  dz is bf16 because the matrix pipe multiplies bf16; in two pieces of it, so that nothing is lost, dX and dW would
// be twice the products.  Against 64 bits dX and dW are 2.4e-3 of their norm off with an activation and 3.0e-3 with a gate too, where the rounding of the results alone is 1.7e-3; db is summed from
// dz as it is before its rounding.
//
// What bounds them is the matrix pipe at the clock that power allows, 2 rows n inputs operations each: 13,312 rows, 3,584 to 2 x 14,336 with a gate take 2.37 ms forward
// (1,150 TFLOP/s), 2.00 for dX and 2.02 for dW (1,360), 32,768 rows, 16,384 to 4,096 with a
// residual 3.22 ms (1,365).  Where there are fewer tiles than compute units the contraction is cut into parts, whose
// fp32 sums a second kernel adds up in their order and finishes (no atomics).
//
// With a gate a tile is of 128 outputs: of each wavefront's 128 rows of W the first 64 are of the gate and the others the same ones of the second half, so that a lane has both of
// an output's values.
#include <math.h>

#include <initializer_list>

#include "ops.h"
#include "product.h"
#include "skrull_linear.h"

namespace {

// ---- activations ----
constexpr float kLog2e = 1.44269504088896340736f;

// P(z), the normal distribution's share below z, and e^(-z^2 / 2).  For z < 0 it is e^(-z^2 / 2) G(-z) with G(a) = erfcx(a / sqrt 2) / 2, of which t times a polynomial in
// t = 1 / (1 + a / 4) is within 1.5e-6 for all a (coefficients by least squares on Chebyshev nodes, weighted towards the largest relative error), however small P(z) is.  The exponential's
// argument is rounded twice, which adds up to 2^-24 z^2 of P(z): its relative error is 1.7e-6 to z = -4, 4e-6 to -8 and 7e-6 to -13, behind which e^(-z^2 / 2) is below fp32's normal numbers.
__device__ __forceinline__ float normal_share(float z, float &density)
{
    const float a = fabsf(z), t = __builtin_amdgcn_rcpf(__builtin_fmaf(a, 0.25f, 1.0f));
    float p = -0.0393727683f;
    p = __builtin_fmaf(p, t, 0.0861844867f);
    p = __builtin_fmaf(p, t, 0.00641432637f);
    p = __builtin_fmaf(p, t, 0.0740136877f);
    p = __builtin_fmaf(p, t, 0.0797690004f);
    p = __builtin_fmaf(p, t, 0.0935138166f);
    p = __builtin_fmaf(p, t, 0.0997414291f);
    p = __builtin_fmaf(p, t, 0.0997354612f);
    density = fast_exp2(z * z * (-0.5f * kLog2e));
    const float tail = p * t * density;
    return z < 0.0f ? tail : 1.0f - tail;
}
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + fast_exp2(z * -kLog2e)); }

__device__ __forceinline__ float relu(float z) { return z < 0.0f ? 0.0f : z; }   // (a NaN stays one)

template <int ACT>
__device__ __forceinline__ float activation(float z)
{
    if constexpr (ACT == SKRULL_LINEAR_RELU) return relu(z);
    if constexpr (ACT == SKRULL_LINEAR_SILU) return z * sigmoid(z);
    if constexpr (ACT == SKRULL_LINEAR_GELU) {
        float density;
        return z * normal_share(z, density);
    }
    return z;
}
// ... and its derivative
template <int ACT>
__device__ __forceinline__ float activation(float z, float &slope)
{
    slope = 1.0f;
    if constexpr (ACT == SKRULL_LINEAR_RELU) {
        slope = z > 0.0f ? 1.0f : z <= 0.0f ? 0.0f : z;   // (a NaN stays one here too: as 0 it would leave gradients that show nothing of it)
        return relu(z);
    }
    if constexpr (ACT == SKRULL_LINEAR_SILU) {
        const float s = sigmoid(z);
        slope = s * (1.0f + z * (1.0f - s));
        return z * s;
    }
    if constexpr (ACT == SKRULL_LINEAR_GELU) {
        float density;
        const float share = normal_share(z, density);
        slope = share + z * density * 0.398942280401432678f;
        return z * share;
    }
    return z;
}

// ---- products ----
enum Kind { kForward, kDx, kDw };

struct LinearArgs {
    const uint16_t *a, *b;       // operands: rows of the weight or (kDw) of x; rows of x, of dz
    int32_t a_stride, b_stride;  // elements between their rows
    int32_t I, J, C;             // rows and columns of the result (gated: of y); the contraction
    int32_t splits, steps;       // parts of the contraction, steps of a part
    // The last `tail` tiles, fewer than there are workgroups after whole rounds of the others, have theirs in parts of tail_steps steps each
    int32_t tail, tail_parts, tail_steps;
    float *slabs;                // with more than one part: [parts][I][J, gated 2 J]; of a tail [tail][tail_parts][tile's rows][its columns, gated of both halves]
    // the result, and of the forward what else it is made of
    uint16_t *out, *z;           // z [I][J, gated 2 J] or null
    const uint16_t *bias, *residual;
    int64_t out_stride, residual_stride;
    int32_t relu;                // max(z, 0) (in kernels without another activation)
};

__device__ __forceinline__ float wide(uint32_t bf16) { return __builtin_bit_cast(float, bf16 << 16); }
__device__ __forceinline__ void wide4(uint2 v, float f[4])
{
    f[0] = wide(v.x & 0xffff);
    f[1] = __builtin_bit_cast(float, v.x & 0xffff0000u);
    f[2] = wide(v.y & 0xffff);
    f[3] = __builtin_bit_cast(float, v.y & 0xffff0000u);
}

template <Kind K, int NA, int NB, int ACT, bool GATED>
__global__ __launch_bounds__(256, 1) void linear_product_kernel(const LinearArgs p)
{
    constexpr bool A_COLS = K != kForward, B_COLS = K == kDw;
    constexpr int kCols = GATED ? 32 * NA : 64 * NA, kRows = 64 * NB;   // of the result, of a tile
    __shared__ __align__(1024) unsigned char lds[2 * kProductBytes<NA, NB>];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave & 1, wn = wave >> 1;
    const int n = lane & 15, g = lane >> 4;
    const uint32_t a_pitch = (uint32_t)p.a_stride * 2, b_pitch = (uint32_t)p.b_stride * 2;
    Operand<A_COLS, NA> A;
    Operand<B_COLS, NB> B;
    A.init(lane, wave, wm, a_pitch, GATED ? 16 * NA : 32 * NA);
    B.init(lane, wave, wn, b_pitch);

    const int mt = (p.J + kCols - 1) / kCols, nt = (p.I + kRows - 1) / kRows, all_steps = (p.C + kStep - 1) / kStep, whole = mt * nt * p.splits - p.tail, parts = p.tail * p.tail_parts;
    // A die has a piece of the whole tiles, then one of the tail's parts, its workgroups take them by turns.
    const int die = blockIdx.x & 7, first = blockIdx.x >> 3, stride = gridDim.x >> 3, per_die = (whole + 7) / 8, parts_per_die = (parts + 7) / 8;
    auto count = [&](int n, int each) { return max(0, min(n - die * each, each) - first + stride - 1) / stride; };
    const int n_whole = count(whole, per_die), n_items = n_whole + count(parts, parts_per_die);
    // Item i of this workgroup: its tile, its part of the contraction, where that begins and how many steps it has.  Tiles in the order of work: blocks of 8 tiles of columns,
    // through all rows; neighbours in it run at the same time on one die and share their operands in its L2.
    struct Item { int m, nn, s, from, steps, tail; };   // tail: of its tile among the tail's, -1: whole, or a part of all tiles' parts
    auto locate = [&](int i) {
        Item t;
        int tile;
        if (i < n_whole) {
            tile = die * per_die + first + i * stride;
            t.s = tile / (mt * nt);
            tile -= t.s * (mt * nt);
            t.tail = -1;
            t.from = t.s * p.steps;
            t.steps = max(0, min(p.steps, all_steps - t.from));
        } else {
            const int k = die * parts_per_die + first + (i - n_whole) * stride;
            t.tail = k / p.tail_parts;
            t.s = k - t.tail * p.tail_parts;
            tile = whole + t.tail;
            t.from = t.s * p.tail_steps;
            t.steps = max(0, min(p.tail_steps, all_steps - t.from));
        }
        const int block = tile / (8 * nt), r = tile - block * (8 * nt), width = min(8, mt - block * 8);
        t.nn = r / width;
        t.m = block * 8 + r - t.nn * width;
        for (int *f : {&t.m, &t.nn, &t.s, &t.from, &t.steps, &t.tail}) *f = __builtin_amdgcn_readfirstlane(*f);
        return t;
    };
    auto open = [&](int i, Source &a, Source &b, int &left, int &a_tail, int &b_tail) {
        const Item t = locate(i);
        const int m = t.m, nn = t.nn;
        left = t.steps;
        const int64_t k0 = (int64_t)t.from * kStep;
        a_tail = b_tail = (int)(p.C - k0);
        const int64_t ap = a_pitch, bp = b_pitch;
        // (to the end of the matrix' last row: what is behind it reads as zero)
        const int64_t a_at = A_COLS ? k0 * ap + (int64_t)m * kCols * 2 : (int64_t)m * kCols * ap + k0 * 2;
        const int64_t b_at = B_COLS ? k0 * bp + (int64_t)nn * kRows * 2 : (int64_t)nn * kRows * bp + k0 * 2;
        const int64_t a_end = A_COLS ? (int64_t)(p.C - 1) * ap + (int64_t)p.J * 2 : ((GATED ? 2 : 1) * (int64_t)p.J - 1) * ap + (int64_t)p.C * 2;
        const int64_t b_end = B_COLS ? (int64_t)(p.C - 1) * bp + (int64_t)p.I * 2 : (int64_t)(p.I - 1) * bp + (int64_t)p.C * 2;
        a = Source{(const unsigned char *)p.a + a_at, a_end - a_at, a_pitch, A_COLS ? kStep * ap : kStep * 2};
        b = Source{(const unsigned char *)p.b + b_at, b_end - b_at, b_pitch, B_COLS ? kStep * bp : kStep * 2};
    };
    Item t = {};
    auto tile_begin = [&](int i) {
        t = locate(i);
        return t.steps;
    };
    auto tile_end = [&](const f32x4 (&acc)[2 * NA][2 * NB]) {
        constexpr int XS = GATED ? NA : 2 * NA;   // blocks of 16 columns of a wavefront
        const int col0 = t.m * kCols + wm * (kCols / 2), row0 = t.nn * kRows + wn * 32 * NB + n;
        if (t.tail >= 0) {
            float *to = p.slabs + ((int64_t)t.tail * p.tail_parts + t.s) * (kRows * 64 * NA) + (wn * 32 * NB + n) * (64 * NA) + wm * (kCols / 2) + 4 * g;
#pragma unroll
            for (int y = 0; y < 2 * NB; ++y)
#pragma unroll
                for (int x = 0; x < 2 * NA; ++x) {
                    SB();
                    *(float4 *)(to + 16 * y * (64 * NA) + 16 * (x % XS) + (x >= XS ? kCols : 0)) =
                        make_float4(result(acc[x][y][0]), result(acc[x][y][1]), result(acc[x][y][2]), result(acc[x][y][3]));
                }
            return;
        }
        if (p.splits > 1) {
            const int width = GATED ? 2 * p.J : p.J;
#pragma unroll
            for (int y = 0; y < 2 * NB; ++y) {
                const int row = row0 + 16 * y;
                float *to = p.slabs + ((int64_t)t.s * p.I + row) * width + col0 + 4 * g;
#pragma unroll
                for (int x = 0; x < 2 * NA; ++x) {
                    SB();
                    const int c = 16 * (x % XS);
                    if (row < p.I && col0 + c + 4 * g < p.J)   // (a whole number of fours)
                        *(float4 *)(to + c + (x >= XS ? p.J : 0)) = make_float4(result(acc[x][y][0]), result(acc[x][y][1]), result(acc[x][y][2]), result(acc[x][y][3]));
                }
            }
            return;
        }
        // (nothing hides the latency of what a tile's end loads, so it loads much at once: 13,312 rows, 3,584 to 3,584 with a residual, 313 us with a block of 16 rows at a time, 288 with
        // all eight; tiles of 256 x 64 have a second one on the unit)
        constexpr int kRowsAhead = NB == 4 ? 2 * NB : 1;   // blocks of 16
        const bool bias = K == kForward && p.bias, residual = K == kForward && p.residual, keep = K == kForward && p.z;
#pragma unroll
        for (int x = 0; x < XS; x += 2) {
            float b[GATED ? 2 : 1][8] = {};   // of both blocks' columns
            if (bias) {
#pragma unroll
                for (int v = 0; v < 2; ++v) {
                    const int c = col0 + 16 * (x + v) + 4 * g;
                    if (c < p.J) {
                        wide4(*(const uint2 *)(p.bias + c), b[0] + 4 * v);
                        if constexpr (GATED) wide4(*(const uint2 *)(p.bias + p.J + c), b[1] + 4 * v);
                    }
                }
            }
            const int stored = col0 + 16 * x + 16 * (g & 1) + 8 * (g >> 1);   // the eight columns that this lane stores
            auto store = [&](uint16_t *to, int64_t row_stride, int row, const float f[8]) {
                const uint4 u = eight_of(f, f + 4);
                if (row < p.I && stored < p.J) *(uint4 *)(to + (int64_t)row * row_stride + stored) = u;
            };
            auto given = [&](int row, int v) {   // of the residual
                const int c = col0 + 16 * (x + v) + 4 * g;
                return row < p.I && c < p.J ? *(const uint2 *)(p.residual + (int64_t)row * p.residual_stride + c) : uint2{};
            };
            uint2 ahead[kRowsAhead][2] = {};
            if (NB == 4 && residual) {
#pragma unroll
                for (int i = 0; i < 2 * kRowsAhead; ++i) ahead[i >> 1][i & 1] = given(row0 + 16 * (i >> 1), i & 1);
            }
#pragma unroll
            for (int y = 0; y < 2 * NB; ++y) {
                SB();
                const int row = row0 + 16 * y;
                uint2 add[2] = {};
                if (residual) {
#pragma unroll
                    for (int v = 0; v < 2; ++v) add[v] = NB == 4 ? ahead[y % kRowsAhead][v] : given(row, v);
                }
                float f[8], z2[8];
#pragma unroll
                for (int v = 0; v < 8; ++v) {
                    f[v] = result(acc[x + (v >> 2)][y][v & 3]) + b[0][v];
                    if constexpr (GATED) z2[v] = result(acc[XS + x + (v >> 2)][y][v & 3]) + b[1][v];
                }
                if (keep) {
                    const int64_t width = GATED ? 2 * (int64_t)p.J : p.J;
                    store(p.z, width, row, f);
                    if constexpr (GATED) store(p.z + p.J, width, row, z2);
                }
                if constexpr (K == kForward) {
#pragma unroll
                    for (int v = 0; v < 8; ++v) {
                        f[v] = activation<ACT>(f[v]);
                        if (ACT == SKRULL_LINEAR_NONE && p.relu) f[v] = relu(f[v]);
                        if constexpr (GATED) f[v] *= z2[v];
                    }
                    if (residual) {
                        float r[8];
                        wide4(add[0], r);
                        wide4(add[1], r + 4);
#pragma unroll
                        for (int v = 0; v < 8; ++v) f[v] += r[v];
                    }
                }
                store(p.out, p.out_stride, row, f);
            }
        }
    };
    product_tiles<A_COLS, B_COLS, NA, NB, !A_COLS, !B_COLS>(lds, A, B, a_pitch, b_pitch, 0, n_items, 1, open, tile_begin, tile_end, GATED ? p.J : 16 * NA);
}

// What follows the sum f of row `row` and columns c .. c + 3 (gated: of both halves).
template <int ACT, bool GATED>
__device__ __forceinline__ void finish(const LinearArgs &p, int64_t row, int c, float f[GATED ? 2 : 1][4])
{
    const int width = GATED ? 2 * p.J : p.J;
#pragma unroll
    for (int half = 0; half < (GATED ? 2 : 1); ++half) {
        if (p.bias) {
            float b[4];
            wide4(*(const uint2 *)(p.bias + half * p.J + c), b);
#pragma unroll
            for (int v = 0; v < 4; ++v) f[half][v] += b[v];
        }
        if (p.z) *(uint2 *)(p.z + row * width + half * p.J + c) = make_uint2(pack_bf16(f[half][0], f[half][1]), pack_bf16(f[half][2], f[half][3]));
    }
    float r[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (p.residual) wide4(*(const uint2 *)(p.residual + row * p.residual_stride + c), r);
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        f[0][v] = activation<ACT>(f[0][v]);
        if (ACT == SKRULL_LINEAR_NONE && p.relu) f[0][v] = relu(f[0][v]);
        if constexpr (GATED) f[0][v] *= f[1][v];
        f[0][v] += r[v];
    }
    *(uint2 *)(p.out + row * p.out_stride + c) = make_uint2(pack_bf16(f[0][0], f[0][1]), pack_bf16(f[0][2], f[0][3]));
}
// The sum of four values of `parts` slabs, in their order.
__device__ __forceinline__ void sum_parts(const float *from, int64_t slab, int parts, float f[4])
{
    float4 t = *(const float4 *)from;
    for (int k = 1; k < parts; k += 8) {
        float4 u[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) u[j] = *(const float4 *)(from + min(k + j, parts - 1) * slab);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (k + j < parts) { t.x += u[j].x; t.y += u[j].y; t.z += u[j].z; t.w += u[j].w; }
    }
    f[0] = t.x; f[1] = t.y; f[2] = t.z; f[3] = t.w;
}
// The parts' sums and what follows them: four columns to a thread.
template <int ACT, bool GATED>
__global__ __launch_bounds__(256) void linear_sums_kernel(const LinearArgs p)
{
    const int width = GATED ? 2 * p.J : p.J, groups = p.J / 4;
    const int64_t slab = (int64_t)p.I * width;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < (int64_t)p.I * groups; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / groups;
        const int c = (int)(i - row * groups) * 4;
        float f[GATED ? 2 : 1][4];
#pragma unroll
        for (int half = 0; half < (GATED ? 2 : 1); ++half) sum_parts(p.slabs + row * width + c + half * p.J, slab, p.splits, f[half]);
        finish<ACT, GATED>(p, row, c, f);
    }
}
// The same of the tail's tiles, of `rows` rows and 256 columns (gated: of 128 and 128): blockIdx.x a tile, blockIdx.y four rows of it (gated: eight).
template <int ACT, bool GATED>
__global__ __launch_bounds__(256) void linear_tail_kernel(const LinearArgs p, int rows)
{
    constexpr int kCols = GATED ? kTile / 2 : kTile, kGroups = kCols / 4;
    const int mt = (p.J + kCols - 1) / kCols, nt = (p.I + rows - 1) / rows, tile = mt * nt - p.tail + blockIdx.x;
    const int block = tile / (8 * nt), r = tile - block * (8 * nt), width = min(8, mt - block * 8), nn = r / width, m = block * 8 + r - nn * width;
    const int in_tile = blockIdx.y * (256 / kGroups) + threadIdx.x / kGroups, c = threadIdx.x % kGroups * 4;
    const int64_t row = (int64_t)nn * rows + in_tile;
    if (row >= p.I || m * kCols + c >= p.J) return;
    const int64_t slab = (int64_t)rows * kTile;
    const float *from = p.slabs + (int64_t)blockIdx.x * p.tail_parts * slab + in_tile * kTile + c;
    float f[GATED ? 2 : 1][4];
#pragma unroll
    for (int half = 0; half < (GATED ? 2 : 1); ++half) sum_parts(from + half * kCols, slab, p.tail_parts, f[half]);
    finish<ACT, GATED>(p, row, m * kCols + c, f);
}

// ---- dz and the sums of its columns ----
struct DzArgs {
    const uint16_t *z, *dy;   // z [rows, outputs, gated 2 outputs]; null: dz is dy, and only its sums are wanted
    uint16_t *dz;             // null: only its sums are wanted
    float *partial;           // [stripes][outputs, gated 2 outputs], or null
    int64_t dy_stride, rows;
    int32_t outputs, each;    // rows of a stripe
};
// A thread has eight columns of y through the rows of a stripe, and of four rows the loads under way.  Memory-bound: 13,312 rows of 2 x 14,336 take 378 us, 5.05 TB/s.
template <int ACT, bool GATED>
__global__ __launch_bounds__(64) void linear_dz_kernel(const DzArgs a)
{
    const int c = (blockIdx.x * 64 + threadIdx.x) * 8, width = GATED ? 2 * a.outputs : a.outputs;
    if (c >= a.outputs) return;
    const int64_t first = (int64_t)blockIdx.y * a.each, end = min(a.rows, first + a.each);
    float sum[GATED ? 2 : 1][8] = {};
    constexpr int AHEAD = 4;
    for (int64_t r0 = first; r0 < end; r0 += AHEAD) {
        uint4 dy[AHEAD], z1[AHEAD], z2[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const int64_t r = min(r0 + j, end - 1);
            dy[j] = *(const uint4 *)(a.dy + r * a.dy_stride + c);
            if (a.z) {
                z1[j] = *(const uint4 *)(a.z + r * width + c);
                if constexpr (GATED) z2[j] = *(const uint4 *)(a.z + r * width + a.outputs + c);
            }
        }
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            if (r0 + j >= end) break;
            float d[8], f[8], other[8], e[8];
            wide4(make_uint2(dy[j].x, dy[j].y), d);
            wide4(make_uint2(dy[j].z, dy[j].w), d + 4);
            if (a.z) {
                wide4(make_uint2(z1[j].x, z1[j].y), f);
                wide4(make_uint2(z1[j].z, z1[j].w), f + 4);
                if constexpr (GATED) {
                    wide4(make_uint2(z2[j].x, z2[j].y), other);
                    wide4(make_uint2(z2[j].z, z2[j].w), other + 4);
                }
#pragma unroll
                for (int v = 0; v < 8; ++v) {
                    float slope;
                    const float y = activation<ACT>(f[v], slope);
                    if constexpr (GATED) {
                        e[v] = d[v] * y;
                        d[v] *= other[v];
                    }
                    d[v] *= slope;
                }
            }
            uint16_t *to = a.dz + (r0 + j) * width + c;
#pragma unroll
            for (int v = 0; v < 8; ++v) sum[0][v] += d[v];
            if (a.dz) *(uint4 *)to = make_uint4(pack_bf16(d[0], d[1]), pack_bf16(d[2], d[3]), pack_bf16(d[4], d[5]), pack_bf16(d[6], d[7]));
            if constexpr (GATED) {
#pragma unroll
                for (int v = 0; v < 8; ++v) sum[1][v] += e[v];
                if (a.dz) *(uint4 *)(to + a.outputs) = make_uint4(pack_bf16(e[0], e[1]), pack_bf16(e[2], e[3]), pack_bf16(e[4], e[5]), pack_bf16(e[6], e[7]));
            }
        }
    }
    if (!a.partial) return;
#pragma unroll
    for (int half = 0; half < (GATED ? 2 : 1); ++half) {
        float4 *to = (float4 *)(a.partial + (int64_t)blockIdx.y * width + half * a.outputs + c);
        to[0] = make_float4(sum[half][0], sum[half][1], sum[half][2], sum[half][3]);
        to[1] = make_float4(sum[half][4], sum[half][5], sum[half][6], sum[half][7]);
    }
}

// db from the stripes' sums, in their order: 64 columns to a workgroup, 16 wavefronts share the stripes.
__global__ __launch_bounds__(1024) void linear_db_kernel(const float *partial, int stripes, int width, uint16_t *db)
{
    __shared__ float part[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
    float s = 0.0f;
    if (c < width) {
#pragma unroll 8
        for (int i = wave; i < stripes; i += 16) s += partial[(int64_t)i * width + c];
    }
    part[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && c < width) {
        s = 0.0f;
#pragma unroll
        for (int k = 0; k < 16; ++k) s += part[k][lane];
        db[c] = (uint16_t)pack_bf16(s, s);
    }
}

// ---- host ----
int check(const skrull_linear_t *p)
{
    if (!p) return refuse("linear: null pointer");
    if (p->rows < 0 || p->rows > 1 << 24) return refuse("linear: %lld rows", (long long)p->rows);
    if (p->inputs < 8 || p->inputs > 65536 || p->inputs % 8 != 0) return refuse("linear: inputs %d is not a multiple of 8 from 8 to 65536", p->inputs);
    if (p->outputs < 8 || p->outputs > 65536 || p->outputs % 8 != 0) return refuse("linear: outputs %d is not a multiple of 8 from 8 to 65536", p->outputs);
    if (p->activation < SKRULL_LINEAR_NONE || p->activation > SKRULL_LINEAR_SILU) return refuse("linear: unknown activation %d", p->activation);
    if (p->gated != 0 && p->gated != 1) return refuse("linear: gated is neither 0 nor 1");
    // (a tile's rows of both halves lie within 31 bits of bytes)
    if (p->gated && ((int64_t)p->outputs + kTile) * p->inputs >= (int64_t)1 << 30) return refuse("linear: gated, %d outputs of %d inputs", p->outputs, p->inputs);
    return SKRULL_OK;
}
// A tensor with rows, for checks.
struct Rows {
    const char *name;
    const void *at;
    int64_t rows, width, stride;
    int64_t bytes() const { return rows > 0 ? ((rows - 1) * stride + width) * 2 : 0; }
};
int check_rows(const Rows &t)
{
    if (!t.at || !aligned_to(t.at, 16)) return refuse("linear: %s is null or misaligned", t.name);
    if (t.stride < t.width || t.stride > 1 << 20 || t.stride % 8 != 0) return refuse("linear: stride %lld of %s", (long long)t.stride, t.name);
    return SKRULL_OK;
}
int check_apart(const Rows &out, std::initializer_list<Rows> others)
{
    for (const Rows &t : others)
        if (out.at && t.at && overlap(out.at, out.bytes(), t.at, t.bytes())) return refuse("linear: %s overlaps %s", out.name, t.name);
    return SKRULL_OK;
}

// Rows and columns of a product's tile / 64, and the parts of its contraction.
struct Shape {
    int na, nb, splits, steps, tail, tail_parts, tail_steps;   // see LinearArgs
};
int tiles_of(int64_t n, int size) { return (int)((n + size - 1) / size); }
// Which tiles, and in how many parts the contraction: what a launch is expected to take, in us, from what tiles of each shape took (37 to 16,384 rows, 896 to 4,096 inputs and
// outputs):
//   tile (columns x rows)   at once on a unit   a step with 1, 2, 3, 4 of them   a tile's start and end
//   256 x 256               1                   1.2 to 1.65 (power)              9
//   256 x 64                2                   0.60  1.03                       5
//   64 x 64 (forward)       4                   0.35  0.40  0.60  0.80           3
// Where tiles are more than workgroups, the last ones, if they are half a round or less, are cut into parts (4,500 rows, 4,096 to 4,096, 288 tiles: the forward takes 179 us with
// all whole and 137 so; 13,312 rows, 3,584 to 28,672, 1,568 tiles of dW: 2,105 and 1,931).  Parts, whose sums are written, read and added by a launch of its own, cost 4 and
// their bytes at 3 MB a us.  In us, each with the parts that suit it best:
//   rows, inputs, outputs   forward: 256 x 256, 256 x 64, 64 x 64   dX: 256 x 256, 256 x 64   dW: 256 x 256, 256 x 64
//   37, 896, 1,152                          13.5  10.6                  14.5  14.2                12.2  11.8
//   1,001, 904, 1,160                 26.5  15.8  12.1                  25.4  16.9                24.4  15.6
//   4,096, 1,024, 1,024               32.9  17.7  18.2                  28.2  16.8                32.4  25.0
//   500, 4,096, 4,096                 38.0  32.3  32.4                  38.7  33.9                23.1  26.8
//   3,000, 2,048, 2,048               45.8  36.6  40.4                  45.2  35.6                44.3  39.2
//   16,384, 896, 1,152                57.1  48.2  58.6                  34.9  46.2                54.8  56.3
//   8,192, 1,024, 4,096               68.3  82.5  109                   73.1  71.6                72.4  85.6
//   2,000, 3,584, 4,608               81.8  89.7  100                   73.8  78.4                57.1  82.3
Shape shape_of(Kind kind, int64_t I, int64_t J, int64_t C, bool gated)
{
    struct Tile { int na, nb, on_a_unit; double step[4], ends; };
    static const Tile tiles[] = {{4, 4, 1, {1.3}, 9.0}, {4, 1, 2, {0.6, 1.03}, 5.0}, {1, 1, 4, {0.35, 0.4, 0.6, 0.8}, 3.0}};
    const int steps = tiles_of(C, kStep);
    Shape best = {4, 4, 1, steps, 0, 1, 0};
    if (I == 0 || C == 0) return best;   // (of no rows: nothing is launched)
    double least = 0.0;
    for (const Tile &t : tiles) {
        if (t.na == 1 && (kind != kForward || gated)) continue;
        const int64_t n = (int64_t)tiles_of(I, 64 * t.nb) * tiles_of(J, (gated ? 32 : 64) * t.na), at_once = (int64_t)t.on_a_unit * kGrid;   // (none of no rows)
        // `items` of `each` steps
        auto time = [&](int64_t items, int each) {
            const int64_t full = items / at_once, rest = items - full * at_once;
            return (double)full * (each * t.step[t.on_a_unit - 1] + t.ends) + (rest ? each * t.step[(rest - 1) / kGrid] + t.ends : 0.0);
        };
        for (int parts = 1; parts <= 16 && parts <= steps; ++parts) {
            const int each = (steps + parts - 1) / parts, real = (steps + each - 1) / each;
            const double sums = real > 1 ? 4.0 * (gated ? 2 : 1) * (double)real * (double)I * (double)J : 0.0;
            if (real < parts || sums > (double)(128 << 20)) continue;
            const double us = time(n * real, each) + (real > 1 ? 4.0 + sums / 3e6 : 0.0);
            if (least == 0.0 || us < least) {
                least = us;
                best = {t.na, t.nb, real, each, 0, 1, 0};
            }
        }
        // whole rounds, and what is left in parts
        const int64_t full = n / at_once;
        const int tail = (int)(n - full * at_once);
        if (t.na == 1 || full == 0 || tail == 0 || 2 * tail > at_once) continue;
        int parts = (int)at_once / tail;
        if (parts > 16) parts = 16;
        if (parts > steps) parts = steps;
        const int each = (steps + parts - 1) / parts, real = (steps + each - 1) / each;
        const double us = time(full * at_once, steps) + time((int64_t)tail * real, each) + 4.0 + (double)tail * real * (64 * t.na * 64 * t.nb * 4) / 3e6;
        if (real > 1 && us < least) {
            least = us;
            best = {t.na, t.nb, 1, steps, tail, real, each};
        }
    }
    return best;
}
int64_t slab_bytes(const Shape &s, int64_t I, int64_t width)
{
    return s.splits > 1 ? (int64_t)s.splits * I * width * 4 : (int64_t)s.tail * s.tail_parts * (64 * s.na) * (64 * s.nb) * 4;
}

// Stripes of dz: 2,048 workgroups of a wavefront, or as many as have 4 rows.  db alone in us, with 1,024, 2,048 and 4,096: 13,312 rows of 2 x 14,336 218, 200, 214; 32,768 of
// 4,096 56, 43, 46; 26,000 of 896 38, 32, 32.
struct Stripes {
    int count, each;
    Stripes(int64_t rows, int outputs)
    {
        const int across = tiles_of(outputs, 512);
        int64_t n = 2048 / across;
        if (n < 1) n = 1;
        if (n > (rows + 3) / 4) n = (rows + 3) / 4;
        if (n < 1) n = 1;
        each = (int)((rows + n - 1) / n);
        if (each < 1) each = 1;
        count = rows > 0 ? (int)((rows + each - 1) / each) : 1;
    }
};
bool plain(const skrull_linear_t &p) { return p.activation == SKRULL_LINEAR_NONE && !p.gated; }

// The workspace, from sizes alone.
struct Layout {
    Shape first, dx, dw;   // first: the forward's product
    Stripes stripes;
    int64_t n, dz, partial, slabs, bytes;
    Layout(const skrull_linear_t &p, bool backward) : stripes(p.rows, p.outputs)
    {
        n = (p.gated ? 2 : 1) * (int64_t)p.outputs;
        bytes = 0;
        auto take = [&](int64_t size) { const int64_t at = bytes; bytes += (size + 255) & ~(int64_t)255; return at; };
        first = shape_of(kForward, p.rows, p.outputs, p.inputs, p.gated != 0);
        dx = shape_of(kDx, p.rows, p.inputs, n, false);
        dw = shape_of(kDw, n, p.inputs, p.rows, false);
        dz = partial = 0;
        if (backward) {
            if (!plain(p)) dz = take(p.rows * n * 2);
            partial = take(stripes.count * n * 4);
            const int64_t a = slab_bytes(dx, p.rows, p.inputs), b = slab_bytes(dw, n, p.inputs);
            slabs = take(a > b ? a : b);
        } else {
            slabs = take(slab_bytes(first, p.rows, n));
        }
    }
};

template <Kind K, int ACT, bool GATED>
hipError_t launch(const Shape &s, const LinearArgs &a, hipStream_t st)
{
    if constexpr (K == kForward && !GATED)
        if (s.na == 1) {
            linear_product_kernel<K, 1, 1, ACT, GATED><<<4 * kGrid, 256, 0, st>>>(a);   // (as many fit the units)
            return hipGetLastError();
        }
    if (s.nb == 1) {
        linear_product_kernel<K, 4, 1, ACT, GATED><<<2 * kGrid, 256, 0, st>>>(a);
        return hipGetLastError();
    }
    linear_product_kernel<K, 4, 4, ACT, GATED><<<kGrid, 256, 0, st>>>(a);
    return hipGetLastError();
}
template <Kind K, int ACT, bool GATED>
hipError_t multiply(const Shape &s, LinearArgs a, hipStream_t st)
{
    a.splits = s.splits;
    a.steps = s.steps;
    a.tail = s.tail;
    a.tail_parts = s.tail_parts;
    a.tail_steps = s.tail_steps;
    hipError_t e = launch<K, ACT, GATED>(s, a, st);
    if (e == hipSuccess && s.splits > 1) {
        const int64_t blocks = ((int64_t)a.I * (a.J / 4) + 255) / 256;
        linear_sums_kernel<ACT, GATED><<<(int)(blocks < 4096 ? blocks : 4096), 256, 0, st>>>(a);
        e = hipGetLastError();
    }
    if (e == hipSuccess && s.tail > 0) {
        const int at_once = 256 / ((GATED ? kTile / 2 : kTile) / 4);
        linear_tail_kernel<ACT, GATED><<<dim3((unsigned)s.tail, (unsigned)(64 * s.nb / at_once)), 256, 0, st>>>(a, 64 * s.nb);
        e = hipGetLastError();
    }
    return e;
}
template <bool GATED>
hipError_t forward(int activation, const Shape &s, const LinearArgs &a, hipStream_t st)
{
    if (activation == SKRULL_LINEAR_GELU) return multiply<kForward, SKRULL_LINEAR_GELU, GATED>(s, a, st);
    if (activation == SKRULL_LINEAR_SILU) return multiply<kForward, SKRULL_LINEAR_SILU, GATED>(s, a, st);
    return multiply<kForward, SKRULL_LINEAR_NONE, GATED>(s, a, st);
}
template <bool GATED>
void form_dz(int activation, dim3 grid, const DzArgs &a, hipStream_t st)
{
    if (activation == SKRULL_LINEAR_RELU) linear_dz_kernel<SKRULL_LINEAR_RELU, GATED><<<grid, 64, 0, st>>>(a);
    else if (activation == SKRULL_LINEAR_GELU) linear_dz_kernel<SKRULL_LINEAR_GELU, GATED><<<grid, 64, 0, st>>>(a);
    else if (activation == SKRULL_LINEAR_SILU) linear_dz_kernel<SKRULL_LINEAR_SILU, GATED><<<grid, 64, 0, st>>>(a);
    else linear_dz_kernel<SKRULL_LINEAR_NONE, GATED><<<grid, 64, 0, st>>>(a);
}

// Zeros (dw and db of no rows).
__global__ __launch_bounds__(256) void linear_zeros_kernel(uint4 *to, int64_t n)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) to[i] = make_uint4(0, 0, 0, 0);
}

}  // namespace

extern "C" {

int64_t skrull_linear_workspace(const skrull_linear_t *p, int backward)
{
    return check(p) == SKRULL_OK ? Layout(*p, backward != 0).bytes : -1;
}

int skrull_linear_fwd(const skrull_linear_t *p, const void *x, const void *w, const void *b, const void *residual, void *y, void *z,
                      void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (int rc = check(p)) return rc;
    if (p->rows == 0) return SKRULL_OK;
    const Layout l(*p, false);
    const Rows tx = {"x", x, p->rows, p->inputs, p->x_stride}, tw = {"w", w, l.n, p->inputs, p->inputs}, tb = {"b", b, 1, l.n, l.n};
    const Rows tr = {"residual", residual, p->rows, p->outputs, p->residual_stride}, ty = {"y", y, p->rows, p->outputs, p->y_stride}, tz = {"z", z, p->rows, l.n, l.n};
    for (const Rows *t : {&tx, &tw, &ty})
        if (int rc = check_rows(*t)) return rc;
    for (const Rows *t : {&tb, &tr, &tz})
        if (t->at)
            if (int rc = check_rows(*t)) return rc;
    if (l.bytes && (!workspace || !aligned_to(workspace, 16) || (int64_t)workspace_bytes < l.bytes))
        return refuse("linear: workspace is null, misaligned or below %lld bytes", (long long)l.bytes);
    const Rows ws = {"workspace", l.bytes ? workspace : nullptr, 1, l.bytes / 2, l.bytes / 2};
    if (int rc = check_apart(ty, {tx, tw, tb, tz, ws})) return rc;
    if (!(y == residual && p->y_stride == p->residual_stride))
        if (int rc = check_apart(ty, {tr})) return rc;
    if (int rc = check_apart(tz, {tx, tw, tb, tr, ws})) return rc;
    if (int rc = check_apart(ws, {tx, tw, tb, tr})) return rc;
    int compute_units = 0;
    if (int rc = current_device(&compute_units)) return rc;
    LinearArgs a = {};
    a.a = (const uint16_t *)w; a.b = (const uint16_t *)x; a.a_stride = p->inputs; a.b_stride = (int32_t)p->x_stride;
    a.I = (int32_t)p->rows; a.J = p->outputs; a.C = p->inputs;
    a.slabs = (float *)((unsigned char *)workspace + l.slabs);
    a.out = (uint16_t *)y; a.z = (uint16_t *)z; a.bias = (const uint16_t *)b; a.residual = (const uint16_t *)residual;
    a.out_stride = p->y_stride; a.residual_stride = p->residual_stride;
    a.relu = p->activation == SKRULL_LINEAR_RELU;
    const hipError_t e = p->gated ? forward<true>(p->activation, l.first, a, (hipStream_t)hip_stream) : forward<false>(p->activation, l.first, a, (hipStream_t)hip_stream);
    return e == hipSuccess ? SKRULL_OK : launch_failed(e, "linear launch");
}

int skrull_linear_bwd(const skrull_linear_t *p, const void *x, const void *w, const void *z, const void *dy, void *dx, void *dw, void *db,
                      void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (int rc = check(p)) return rc;
    if (!dx && !dw && !db) return SKRULL_OK;
    const Layout l(*p, true);
    const Rows tx = {"x", x, p->rows, p->inputs, p->x_stride}, tw = {"w", w, l.n, p->inputs, p->inputs}, tz = {"z", z, p->rows, l.n, l.n};
    const Rows tdy = {"dy", dy, p->rows, p->outputs, p->dy_stride}, tdx = {"dx", dx, p->rows, p->inputs, p->inputs}, tdw = {"dw", dw, l.n, p->inputs, p->inputs};
    const Rows tdb = {"db", db, 1, l.n, l.n};
    for (const Rows *t : {&tdx, &tdw, &tdb})
        if (t->at)
            if (int rc = check_rows(*t)) return rc;
    hipStream_t st = (hipStream_t)hip_stream;
    int compute_units = 0;
    if (p->rows == 0) {
        if (dw && db)
            if (int rc = check_apart(tdw, {tdb})) return rc;
        if (int rc = current_device(&compute_units)) return rc;
        if (dw) linear_zeros_kernel<<<256, 256, 0, st>>>((uint4 *)dw, l.n * p->inputs / 8);
        if (db) linear_zeros_kernel<<<1, 256, 0, st>>>((uint4 *)db, l.n / 8);
        const hipError_t e = hipGetLastError();
        return e == hipSuccess ? SKRULL_OK : launch_failed(e, "linear launch");
    }
    const bool direct = plain(*p);   // dz is dy
    for (const Rows *t : {&tx, &tw, &tdy})
        if (int rc = check_rows(*t)) return rc;
    if (!direct)
        if (int rc = check_rows(tz)) return rc;
    if (!workspace || !aligned_to(workspace, 16) || (int64_t)workspace_bytes < l.bytes)
        return refuse("linear: workspace is null, misaligned or below %lld bytes", (long long)l.bytes);
    const Rows ws = {"workspace", workspace, 1, l.bytes / 2, l.bytes / 2}, kept = direct ? Rows{} : tz;
    if (int rc = check_apart(tdx, {tx, tw, kept, tdy, tdw, tdb, ws})) return rc;
    if (int rc = check_apart(tdw, {tx, tw, kept, tdy, tdb, ws})) return rc;
    if (int rc = check_apart(tdb, {tx, tw, kept, tdy, ws})) return rc;
    if (int rc = check_apart(ws, {tx, tw, kept, tdy})) return rc;
    if (int rc = current_device(&compute_units)) return rc;
    unsigned char *scratch = (unsigned char *)workspace;
    hipError_t e = hipSuccess;
    const uint16_t *dz = (const uint16_t *)dy;
    int32_t dz_stride = (int32_t)p->dy_stride;
    if (!direct || db) {
        DzArgs a = {};
        a.dy = (const uint16_t *)dy; a.dy_stride = p->dy_stride; a.rows = p->rows; a.outputs = p->outputs; a.each = l.stripes.each;
        if (!direct) {
            a.z = (const uint16_t *)z;
            a.dz = dx || dw ? (uint16_t *)(scratch + l.dz) : nullptr;
            dz = (const uint16_t *)(scratch + l.dz);
            dz_stride = (int32_t)l.n;
        }
        a.partial = db ? (float *)(scratch + l.partial) : nullptr;
        const dim3 grid((unsigned)tiles_of(p->outputs, 512), (unsigned)l.stripes.count);
        if (p->gated) form_dz<true>(p->activation, grid, a, st);
        else form_dz<false>(p->activation, grid, a, st);
        e = hipGetLastError();
        if (e == hipSuccess && db) {
            linear_db_kernel<<<(int)((l.n + 63) / 64), 1024, 0, st>>>(a.partial, l.stripes.count, (int)l.n, (uint16_t *)db);
            e = hipGetLastError();
        }
    }
    LinearArgs a = {};
    a.slabs = (float *)(scratch + l.slabs);
    a.out_stride = p->inputs;
    a.J = p->inputs;
    a.b = dz; a.b_stride = dz_stride;
    if (e == hipSuccess && dx) {
        a.a = (const uint16_t *)w; a.a_stride = p->inputs;
        a.I = (int32_t)p->rows; a.C = (int32_t)l.n;
        a.out = (uint16_t *)dx;
        e = multiply<kDx, SKRULL_LINEAR_NONE, false>(l.dx, a, st);
    }
    if (e == hipSuccess && dw) {
        a.a = (const uint16_t *)x; a.a_stride = (int32_t)p->x_stride;
        a.I = (int32_t)l.n; a.C = (int32_t)p->rows;
        a.out = (uint16_t *)dw;
        e = multiply<kDw, SKRULL_LINEAR_NONE, false>(l.dw, a, st);
    }
    return e == hipSuccess ? SKRULL_OK : launch_failed(e, "linear launch");
}

}  // extern "C"
