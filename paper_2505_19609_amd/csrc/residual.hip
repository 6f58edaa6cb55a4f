// The residual stream between two blocks, forward and backward (include/skrull_residual.h).
//
// What bounds it: memory.  The forward reads r and z and writes the new stream and y, the backward reads r, z and two gradients and writes two, each once: as in
// norm.hip a row stays in the registers of its lanes from its loads to its stores, and the next row is asked for before this one is summed.  32,768 rows of 4,096 bf16
// with both norms and all vectors: 214 us forward (5.0 TB/s), 304 backward (5.3), 8 the vectors' sums.
//
// Both norms come down to two sums over a row each way, one after the other, since the second norm is of what the first one gives.  The five vectors' gradients
// come down to four sums over the rows: with c1 = gate * post_w and n = h1 post_w + post_b
//     A = sum dy h2 = dw,  B = sum dy = db,  E1 = sum e h1,  E0 = sum e:   dgate = post_w E1 + post_b E0,  dpost_w = gate E1,  dpost_b = gate E0
// so a column takes four accumulators.  They are added up over the workgroups by a second kernel in a fixed order (no atomics).
//
// A row belongs to as few wavefronts as give each lane one piece of 8 columns: 1 (up to 512 columns), 2, 4, 8 or 16 (up to 8,192).  What the backward
// keeps of a column (three vectors' values, four sums, two gradients, the row's two normed values, four loads under way) fits 128 registers that way.
#include <hip/hip_runtime.h>

#include <math.h>

#include <initializer_list>
#include <utility>

#include "ops.h"
#include "rows.h"
#include "skrull_residual.h"

namespace {

struct ResidualArgs {
    const void *r, *z, *w, *b, *post_w, *post_b, *gate;
    const void *d_r_out, *dy;   // null: no gradient comes that way
    void *r_out, *y;            // dr, dz
    float *stats;               // [4][rows], or null
    float *partial;             // [workgroups][4][cols], or null
    int64_t r_stride, z_stride, d_r_out_stride, dy_stride, r_out_stride, y_stride;
    int64_t rows;
    int32_t cols, weight_type;
    float eps, inv_cols, scale;
};

constexpr int threads_of(int waves) { return waves == 1 ? 256 : 64 * waves; }   // (one wavefront to a row: four rows at a time)

// gate * post_w and gate * post_b of this lane's columns, zero where they are not its own: what the normed z is multiplied by and what is added
template <bool SMALL>
__device__ __forceinline__ void load_post(const ResidualArgs &a, const Columns<SMALL> &k, float c1[8], float c0[8])
{
    float gate[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) gate[i] = k.has(i) ? 1.0f : 0.0f;
    if (a.gate) load_weight(a.gate, a.weight_type, k, gate);
#pragma unroll
    for (int i = 0; i < 8; ++i) c1[i] = 1.0f, c0[i] = 0.0f;
    if (a.post_w) load_weight(a.post_w, a.weight_type, k, c1);
    if (a.post_b) load_weight(a.post_b, a.weight_type, k, c0);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        c1[i] *= gate[i];
        c0[i] *= gate[i];
    }
}

// A row's address, the same for all lanes: what is loaded or stored is that and 32 bits of each lane's own.  (Left to the compiler, each tensor has a 64-bit address in every
// lane through the loop, and with 16 wavefronts the backward's registers do not suffice.)
typedef unsigned char __attribute__((address_space(1))) *row_t;
__device__ __forceinline__ row_t row_at(const void *base, int64_t row, int64_t stride, int size)
{
    uint64_t at = (uint64_t)base + (uint64_t)(row * stride) * size;
    asm volatile("" : "+s"(at));
    return (row_t)at;
}

// This lane's piece of a row.  Every lane loads one, those without columns the row's last, so that nothing depends on the lane (SMALL: value by value).
template <class T, bool SMALL>
struct Piece {
    typename T::Raw raw;
    __device__ __forceinline__ void fetch(row_t row, const Columns<SMALL> &k)
    {
        const typename T::type *p = (const typename T::type *)(row + (uint32_t)k.first * (uint32_t)sizeof(typename T::type));
        if constexpr (SMALL) raw = T::load_some(p, 8 - k.skip);
        else raw = T::load8(p);
    }
    __device__ __forceinline__ void get(const Columns<SMALL> &k, float f[8]) const
    {
        T::widen(raw, f);
        if constexpr (!SMALL) {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = k.has(i) ? f[i] : 0.0f;
        }
    }
};
template <class T, bool SMALL>
__device__ __forceinline__ void store_row(row_t row, const Columns<SMALL> &k, const float f[8])
{
    store_piece<T, SMALL>((typename T::type *)row, k, f);
}
template <bool SMALL>
__device__ __forceinline__ void init_columns(Columns<SMALL> &k, int lane, int lanes, int cols)
{
    k.init(0, lane, lanes, cols);
    if (!SMALL && k.skip == 8) k.first = cols - 8;
}

// x and the values of the lanes that differ in one bit, summed bit by bit: without addresses for the exchange and, but for the last two, without a wait.
template <int CONTROL>
__device__ __forceinline__ float add_dpp(float x)
{
    return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CONTROL, 0xf, 0xf, true));
}
__device__ __forceinline__ float wave_sum(float x)
{
    x = add_dpp<0xb1>(x);    // lanes 1 0 3 2 of each four
    x = add_dpp<0x4e>(x);    // 2 3 0 1
    x = add_dpp<0x141>(x);   // each eight in reverse: the other four
    x = add_dpp<0x140>(x);   // each sixteen in reverse: the other eight
    float r, t;              // (written out, as add_other_half in tiles.h)
    asm volatile("v_mov_b32 %0, %2\n\tv_mov_b32 %1, %2\n\ts_nop 1\n\tv_permlane16_swap_b32 %0, %1\n\tv_add_f32 %0, %0, %1\n\t"
                 "v_mov_b32 %1, %0\n\ts_nop 1\n\tv_permlane32_swap_b32 %0, %1\n\tv_add_f32 %0, %0, %1"
                 : "=&v"(r), "=&v"(t) : "v"(x));
    return r;
}
// Sums of N values over the lanes of a row, in every lane.  `lds`: room for 2 x WAVES x N floats, used by turns.
template <int WAVES, int N>
__device__ __forceinline__ void sums_of_row(float v[N], float *lds, int &turn)
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
    if constexpr (WAVES > 1) {
        float *mine = lds + turn * (WAVES * N);
        turn ^= 1;   // (the next sums use the other half, so one barrier is enough)
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) mine[wave * N + i] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float s = 0.0f;
#pragma unroll
            for (int k = 0; k < WAVES; ++k) s += mine[k * N + i];
            v[i] = s;
        }
    }
}

// x less its mean (CENTER) in the lanes' own columns, zero in others; returns 1 / its deviation.
template <int WAVES, bool CENTER, bool SMALL>
__device__ __forceinline__ float centred(float x[8], const Columns<SMALL> &k, const ResidualArgs &a, float *lds, int &turn, float &mean)
{
    mean = 0.0f;
    if constexpr (CENTER) {
        float s[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < 8; ++i) s[0] += x[i];
        sums_of_row<WAVES, 1>(s, lds, turn);
        mean = s[0] * a.inv_cols;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = k.has(i) ? x[i] - mean : 0.0f;
    }
    float q[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < 8; ++i) q[0] += x[i] * x[i];
    sums_of_row<WAVES, 1>(q, lds, turn);
    return 1.0f / sqrtf(q[0] * a.inv_cols + a.eps);
}

template <class T, class R, int WAVES, bool CENTER, bool POST, bool SMALL>
__global__ __launch_bounds__(threads_of(WAVES)) void residual_fwd_kernel(const ResidualArgs a)
{
    constexpr int ROWS = WAVES == 1 ? 4 : 1;   // rows of a workgroup at a time
    __shared__ float lds[2 * WAVES];
    int turn = 0;
    const int slot = ROWS > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0, lane = ROWS > 1 ? threadIdx.x & 63 : threadIdx.x;
    float w[8], b[8], c1[8], c0[8];
    Columns<SMALL> col;
    init_columns(col, lane, 64 * WAVES, a.cols);
    load_weight(a.w, a.weight_type, col, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = 0.0f;
    if (a.b) load_weight(a.b, a.weight_type, col, b);
    load_post(a, col, c1, c0);
    constexpr int TS = sizeof(typename T::type), RS = sizeof(typename R::type);
    const int64_t stride = (int64_t)gridDim.x * ROWS;
    int64_t row = (int64_t)blockIdx.x * ROWS + slot;   // (a wavefront to a row, or all of them: no wavefront waits for one that has left)
    Piece<T, SMALL> next_z;
    Piece<R, SMALL> next_r;
    auto fetch = [&](int64_t i) {
        next_z.fetch(row_at(a.z, i, a.z_stride, TS), col);
        next_r.fetch(row_at(a.r, i, a.r_stride, RS), col);
    };
    fetch(min(row, a.rows - 1));
    for (; row < a.rows; row += stride) {
        float z[8], r[8];
        next_z.get(col, z);
        next_r.get(col, r);
        fetch(min(row + stride, a.rows - 1));   // (the last row once more rather than under a condition)
        float mean1 = 0.0f, rstd1 = 1.0f, mean2;
        if constexpr (POST) rstd1 = centred<WAVES, CENTER>(z, col, a, lds, turn, mean1);
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = r[i] * a.scale + (z[i] * rstd1 * c1[i] + c0[i]);
        store_row<R>(row_at(a.r_out, row, a.r_out_stride, RS), col, x);
        const float rstd2 = centred<WAVES, CENTER>(x, col, a, lds, turn, mean2);
        if (lane == 0 && a.stats) {
            float *s = a.stats + row;
            if (POST && CENTER) s[0] = mean1;
            if (POST) s[a.rows] = rstd1;
            if (CENTER) s[2 * a.rows] = mean2;
            s[3 * a.rows] = rstd2;
        }
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = x[i] * rstd2 * w[i] + b[i];
        store_row<T>(row_at(a.y, row, a.y_stride, TS), col, y);
    }
}

template <class T, class R, int WAVES, bool CENTER, bool POST, bool SMALL>
__global__ __launch_bounds__(threads_of(WAVES)) void residual_bwd_kernel(const ResidualArgs a)
{
    constexpr int ROWS = WAVES == 1 ? 4 : 1;
    __shared__ float lds[2 * WAVES * 2];
    int turn = 0;
    const int slot = ROWS > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0, lane = ROWS > 1 ? threadIdx.x & 63 : threadIdx.x;
    // A, B, E1, E0.  With 16 wavefronts they lie in LDS, for the registers' sake: 256 bytes a lane and row, a tenth of what LDS can do in the row's time.
    constexpr bool IN_LDS = WAVES == 16;
    __shared__ float4 lds_sum[IN_LDS ? 4 : 1][2][IN_LDS ? 1024 : 1];
    float w[8], c1[8], c0[8], sum[4][8];
    Columns<SMALL> col;
    init_columns(col, lane, 64 * WAVES, a.cols);
    load_weight(a.w, a.weight_type, col, w);
    load_post(a, col, c1, c0);
    auto add = [&](int k, const float f[8]) {
        if constexpr (IN_LDS) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                float4 &s = lds_sum[k][half][lane];
                s = make_float4(s.x + f[4 * half], s.y + f[4 * half + 1], s.z + f[4 * half + 2], s.w + f[4 * half + 3]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[k][i] += f[i];
        }
    };
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if constexpr (IN_LDS) lds_sum[k][0][lane] = lds_sum[k][1][lane] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[k][i] = 0.0f;
    }
    constexpr int TS = sizeof(typename T::type), RS = sizeof(typename R::type);
    const int64_t stride = (int64_t)gridDim.x * ROWS;
    int64_t row = (int64_t)blockIdx.x * ROWS + slot;
    Piece<T, SMALL> next_z, next_dy = {};
    Piece<R, SMALL> next_r, next_ds = {};
    float next_stats[4] = {0.0f, 1.0f, 0.0f, 0.0f};
    constexpr bool AHEAD = WAVES < 16;   // (with 16 wavefronts, of 128 registers each, there is no room for it)
    auto fetch = [&](int64_t i) {
        next_z.fetch(row_at(a.z, i, a.z_stride, TS), col);
        next_r.fetch(row_at(a.r, i, a.r_stride, RS), col);
        if (a.dy) next_dy.fetch(row_at(a.dy, i, a.dy_stride, TS), col);
        if (a.d_r_out) next_ds.fetch(row_at(a.d_r_out, i, a.d_r_out_stride, RS), col);
        const float *s = a.stats + i;
        if (POST && CENTER) next_stats[0] = s[0];
        if (POST) next_stats[1] = s[a.rows];
        if (CENTER) next_stats[2] = s[2 * a.rows];
        next_stats[3] = s[3 * a.rows];
    };
    if (AHEAD) fetch(min(row, a.rows - 1));
    for (; row < a.rows; row += stride) {
        if (!AHEAD) fetch(row);
        const float mean1 = next_stats[0], rstd1 = next_stats[1], mean2 = next_stats[2], rstd2 = next_stats[3];
        float h1[8], h2[8], g[8], e[8];
        next_z.get(col, h1);
        next_r.get(col, h2);
        next_dy.get(col, g);
        next_ds.get(col, e);
        if (AHEAD) fetch(min(row + stride, a.rows - 1));
        float s[2] = {0.0f, 0.0f};   // sum g2 h2, sum g2
        float d[8];
        if (CENTER) add(1, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (POST) h1[i] = (CENTER ? h1[i] - mean1 : h1[i]) * rstd1;
            h2[i] = h2[i] * a.scale + (h1[i] * c1[i] + c0[i]);   // (as the forward has it)
            h2[i] = (CENTER ? h2[i] - mean2 : h2[i]) * rstd2;
            d[i] = g[i] * h2[i];
            g[i] *= w[i];   // (zero behind the last column, whatever h2 is there)
            s[0] += g[i] * h2[i];
            if (CENTER) s[1] += g[i];
        }
        add(0, d);
        sums_of_row<WAVES, CENTER ? 2 : 1>(s, lds, turn);
        float m0 = s[0] * a.inv_cols, m1 = CENTER ? s[1] * a.inv_cols : 0.0f;
        s[0] = s[1] = 0.0f;      // sum g1 h1, sum g1
        float dr[8], dz[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            e[i] += (g[i] - m1 - h2[i] * m0) * rstd2;
            dr[i] = e[i] * a.scale;
            d[i] = e[i] * h1[i];
            dz[i] = e[i] * c1[i];
            if (POST) {
                s[0] += dz[i] * h1[i];
                if (CENTER) s[1] += dz[i];
            }
        }
        add(2, d);
        if (CENTER) add(3, e);
        store_row<R>(row_at(a.r_out, row, a.r_out_stride, RS), col, dr);
        if constexpr (POST) {
            sums_of_row<WAVES, CENTER ? 2 : 1>(s, lds, turn);
            m0 = s[0] * a.inv_cols;
            m1 = CENTER ? s[1] * a.inv_cols : 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) dz[i] = (dz[i] - m1 - h1[i] * m0) * rstd1;
        }
        store_row<T>(row_at(a.y, row, a.y_stride, TS), col, dz);
    }
    if (!a.partial) return;
    float *line = a.partial + (int64_t)blockIdx.x * 4 * a.cols;
    if constexpr (ROWS == 1) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (CENTER || k % 2 == 0) {
                if constexpr (IN_LDS) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum[k][i] = ((const float *)&lds_sum[k][i / 4][lane])[i % 4];
                }
                store_piece<Fp32, SMALL>(line + k * a.cols, col, sum[k]);
            }
    } else {   // the wavefronts' own sums first
        __shared__ float sums[ROWS][8][64];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (!CENTER && k % 2) continue;
            if (k) __syncthreads();
#pragma unroll
            for (int i = 0; i < 8; ++i) sums[slot][i][lane] = sum[k][i];
            __syncthreads();
            if (slot == 0) {
                float f[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] = (sums[0][i][lane] + sums[1][i][lane]) + (sums[2][i][lane] + sums[3][i][lane]);
                store_piece<Fp32, SMALL>(line + k * a.cols, col, f);
            }
        }
    }
}

// The vectors' gradients from the partial sums: 64 columns to a workgroup, 16 wavefronts share the lines, in the order of their number.  blockIdx.y: 0 for dw and db, 1
// for the others.
struct SumsArgs {
    const float *partial;
    const void *post_w, *post_b, *gate;
    void *dw, *db, *dpost_w, *dpost_b, *dgate;
    int32_t lines, cols, weight_type, center;
};
__device__ __forceinline__ float weight_at(const void *w, int c, int type, float none)
{
    if (!w) return none;
    return type == SKRULL_TYPE_BF16 ? __builtin_bit_cast(float, (uint32_t)((const uint16_t *)w)[c] << 16) : ((const float *)w)[c];
}
__device__ __forceinline__ void put_weight(void *w, int c, int type, float f)
{
    if (!w) return;
    if (type == SKRULL_TYPE_BF16) ((uint16_t *)w)[c] = to_bf16(f);
    else ((float *)w)[c] = f;
}
__global__ __launch_bounds__(1024) void residual_sums_kernel(const SumsArgs a)
{
    __shared__ float part[2][16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
    if (blockIdx.y ? !a.dpost_w && !a.dpost_b && !a.dgate : !a.dw && !a.db) return;   // (the whole workgroup)
    float s[2] = {0.0f, 0.0f};
    if (c < a.cols) {
        const float *p = a.partial + (int64_t)blockIdx.y * 2 * a.cols + c;
#pragma unroll 4
        for (int i = wave; i < a.lines; i += 16) {
            s[0] += p[(int64_t)i * 4 * a.cols];
            if (a.center) s[1] += p[((int64_t)i * 4 + 1) * a.cols];
        }
    }
    part[0][wave][lane] = s[0];
    part[1][wave][lane] = s[1];
    __syncthreads();
    if (wave == 0 && c < a.cols) {
        s[0] = s[1] = 0.0f;
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            s[0] += part[0][k][lane];
            s[1] += part[1][k][lane];
        }
        if (blockIdx.y == 0) {
            put_weight(a.dw, c, a.weight_type, s[0]);
            put_weight(a.db, c, a.weight_type, s[1]);
        } else {
            const float gate = weight_at(a.gate, c, a.weight_type, 1.0f);
            put_weight(a.dgate, c, a.weight_type, weight_at(a.post_w, c, a.weight_type, 1.0f) * s[0] + (a.post_b ? weight_at(a.post_b, c, a.weight_type, 0.0f) * s[1] : 0.0f));
            put_weight(a.dpost_w, c, a.weight_type, gate * s[0]);
            put_weight(a.dpost_b, c, a.weight_type, gate * s[1]);
        }
    }
}

int check(const skrull_residual_t *p)
{
    if (!p) return refuse("residual: null pointer");
    if (p->rows < 0 || p->rows > INT32_MAX) return refuse("residual: %lld rows", (long long)p->rows);
    if (p->cols < 1 || p->cols > SKRULL_NORM_MAX_COLS) return refuse("residual: %d columns, at most %d", p->cols, SKRULL_NORM_MAX_COLS);
    if (p->kind != SKRULL_NORM_RMS && p->kind != SKRULL_NORM_LAYER) return refuse("residual: unknown kind %d", p->kind);
    if (p->type != SKRULL_TYPE_BF16 && p->type != SKRULL_TYPE_FP32) return refuse("residual: unknown type %d", p->type);
    if (p->residual_type != p->type && p->residual_type != SKRULL_TYPE_FP32) return refuse("residual: residual_type %d with type %d", p->residual_type, p->type);
    if (p->weight_type != SKRULL_TYPE_BF16 && p->weight_type != SKRULL_TYPE_FP32) return refuse("residual: unknown weight_type %d", p->weight_type);
    if (!isfinite(p->eps) || !(p->eps >= 0.0f)) return refuse("residual: eps must be finite and not negative");
    if (!isfinite(p->scale)) return refuse("residual: scale must be finite");
    return SKRULL_OK;
}

// The rows of a tensor, for checks.
struct Rows {
    const char *name;
    const void *at;
    int64_t stride;
    int type;
    int64_t bytes(const skrull_residual_t *p) const { return ((p->rows - 1) * stride + p->cols) * size_of(type); }
};
int check_rows(const Rows &t, const skrull_residual_t *p)
{
    if (!t.at || !aligned_to(t.at, size_of(t.type))) return refuse("residual: %s is null or misaligned", t.name);
    if (t.stride < p->cols || t.stride > INT64_MAX / 8 / (p->rows + 1)) return refuse("residual: stride of %s", t.name);
    return SKRULL_OK;
}
int check_apart(const Rows &a, const Rows &b, const skrull_residual_t *p)
{
    if (a.at && b.at && overlap(a.at, a.bytes(p), b.at, b.bytes(p))) return refuse("residual: %s overlaps %s", a.name, b.name);
    return SKRULL_OK;
}
int check_vectors(std::initializer_list<std::pair<const char *, const void *>> vectors, const skrull_residual_t *p)
{
    for (const auto &v : vectors)
        if (!aligned_to(v.second, size_of(p->weight_type))) return refuse("residual: %s is misaligned", v.first);
    return SKRULL_OK;
}

int waves_of(int cols) { return cols <= 512 ? 1 : cols <= 1024 ? 2 : cols <= 2048 ? 4 : cols <= 4096 ? 8 : 16; }
int rows_of(int waves) { return waves == 1 ? 4 : 1; }

// Workgroups, each with a line of partial sums in the backward: 8 wavefronts to a compute unit (16 where a row has them).  With the next row of each under way that
// keeps the memory busy, and more of them only spread the accesses.  Forward and backward in us, 8, 16 and 32 to a unit (bf16):
//   32,768 x 4,096     183  194  204     289  316  326
//   65,536 x 2,048     187  208  215     306  330  352
//   200,000 x 512      144  165  170     236  246  260
//   26,000 x 896        32   32   33      66   68   89
//   8,192 x 8,192      116   94   96     211  156  165
// Few rows: in the backward a workgroup has `least` = 2 of each wavefront's at least, since the second kernel reads a line of each (both kernels: 932 x 896 14.9 us with one, 11.7 with
// two, 11.4 with four; 300 x 896 9.2, 8.5, 9.2; 500 x 4,096 12.9, 12.7, 13.6).
constexpr int kComputeUnits = 256;
int64_t blocks_of(const skrull_residual_t *p, int least)
{
    const int waves = waves_of(p->cols), rows = rows_of(waves);
    const int64_t most = kComputeUnits * (waves == 16 ? 1 : 8 / (waves == 1 ? 4 : waves)), need = (p->rows + rows * least - 1) / (rows * least);
    return need < most ? need : most;
}

template <class T, class R, bool CENTER, bool POST>
void launch(bool backward, const ResidualArgs &a, int blocks, hipStream_t st)
{
    const int cols = a.cols;
#define SKRULL_RESIDUAL_CASE(WAVES, SMALL)                                                                                  \
    do {                                                                                                                    \
        if (backward) residual_bwd_kernel<T, R, WAVES, CENTER, POST, SMALL><<<blocks, threads_of(WAVES), 0, st>>>(a);       \
        else residual_fwd_kernel<T, R, WAVES, CENTER, POST, SMALL><<<blocks, threads_of(WAVES), 0, st>>>(a);                \
    } while (0)
    if (cols < 8) SKRULL_RESIDUAL_CASE(1, true);
    else if (cols <= 512) SKRULL_RESIDUAL_CASE(1, false);
    else if (cols <= 1024) SKRULL_RESIDUAL_CASE(2, false);
    else if (cols <= 2048) SKRULL_RESIDUAL_CASE(4, false);
    else if (cols <= 4096) SKRULL_RESIDUAL_CASE(8, false);
    else SKRULL_RESIDUAL_CASE(16, false);
#undef SKRULL_RESIDUAL_CASE
}
template <class T, class R>
void launch(bool backward, const skrull_residual_t *p, const ResidualArgs &a, int blocks, hipStream_t st)
{
    if (p->kind == SKRULL_NORM_LAYER) {
        if (a.post_w) launch<T, R, true, true>(backward, a, blocks, st);
        else launch<T, R, true, false>(backward, a, blocks, st);
    } else {
        if (a.post_w) launch<T, R, false, true>(backward, a, blocks, st);
        else launch<T, R, false, false>(backward, a, blocks, st);
    }
}
void launch(bool backward, const skrull_residual_t *p, const ResidualArgs &a, int blocks, hipStream_t st)
{
    if (p->type == SKRULL_TYPE_FP32) launch<Fp32, Fp32>(backward, p, a, blocks, st);
    else if (p->residual_type == SKRULL_TYPE_FP32) launch<Bf16, Fp32>(backward, p, a, blocks, st);
    else launch<Bf16, Bf16>(backward, p, a, blocks, st);
}

ResidualArgs args_of(const skrull_residual_t *p, const void *r, const void *z, const void *w, const void *post_w, const void *post_b, const void *gate)
{
    ResidualArgs a = {};
    a.r = r; a.z = z; a.w = w; a.post_w = post_w; a.post_b = post_b; a.gate = gate;
    a.r_stride = p->r_stride; a.z_stride = p->z_stride; a.rows = p->rows; a.cols = p->cols; a.weight_type = p->weight_type;
    a.eps = p->eps; a.inv_cols = 1.0f / (float)p->cols; a.scale = p->scale;
    return a;
}

}  // namespace

extern "C" {

int skrull_residual_fwd(const skrull_residual_t *p, const void *r, const void *z, const void *w, const void *b, const void *post_w,
                        const void *post_b, const void *gate, void *r_out, void *y, float *stats, void *hip_stream)
{
    if (int rc = check(p)) return rc;
    if ((b || post_b) && p->kind == SKRULL_NORM_RMS) return refuse("residual: no bias without a mean (SKRULL_NORM_RMS)");
    if (post_b && !post_w) return refuse("residual: post_b without post_w");
    if (p->rows == 0) return SKRULL_OK;
    const Rows in_r = {"r", r, p->r_stride, p->residual_type}, in_z = {"z", z, p->z_stride, p->type};
    const Rows out_r = {"r_out", r_out, p->r_out_stride, p->residual_type}, out_y = {"y", y, p->y_stride, p->type};
    for (const Rows *t : {&in_r, &in_z, &out_r, &out_y})
        if (int rc = check_rows(*t, p)) return rc;
    if (!w) return refuse("residual: w is null");
    if (int rc = check_vectors({{"w", w}, {"b", b}, {"post_w", post_w}, {"post_b", post_b}, {"gate", gate}}, p)) return rc;
    if (!aligned_to(stats, 4)) return refuse("residual: stats is misaligned");
    if (!(r_out == r && p->r_out_stride == p->r_stride))
        if (int rc = check_apart(out_r, in_r, p)) return rc;
    if (!(y == z && p->y_stride == p->z_stride))
        if (int rc = check_apart(out_y, in_z, p)) return rc;
    if (int rc = check_apart(out_r, in_z, p)) return rc;
    if (int rc = check_apart(out_y, in_r, p)) return rc;
    if (int rc = check_apart(out_r, out_y, p)) return rc;
    int compute_units = 0;
    if (int rc = current_device(&compute_units)) return rc;
    ResidualArgs a = args_of(p, r, z, w, post_w, post_b, gate);
    a.b = b; a.r_out = r_out; a.y = y; a.stats = stats;
    a.r_out_stride = p->r_out_stride; a.y_stride = p->y_stride;
    launch(false, p, a, (int)blocks_of(p, 1), (hipStream_t)hip_stream);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SKRULL_OK : launch_failed(e, "residual launch");
}

int64_t skrull_residual_workspace(const skrull_residual_t *p)
{
    return check(p) == SKRULL_OK ? blocks_of(p, 2) * 4 * p->cols * 4 + 16 : 0;
}

int skrull_residual_bwd(const skrull_residual_t *p, const void *r, const void *z, const void *w, const void *post_w, const void *post_b,
                        const void *gate, const float *stats, const void *d_r_out, const void *dy, void *dr, void *dz, void *dw, void *db,
                        void *dpost_w, void *dpost_b, void *dgate, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (int rc = check(p)) return rc;
    if ((post_b || db || dpost_b) && p->kind == SKRULL_NORM_RMS) return refuse("residual: no bias without a mean (SKRULL_NORM_RMS)");
    if (post_b && !post_w) return refuse("residual: post_b without post_w");
    if ((dpost_w || dpost_b) && !post_w) return refuse("residual: a gradient of post_w or post_b without post_w");
    if (int rc = check_vectors({{"w", w}, {"post_w", post_w}, {"post_b", post_b}, {"gate", gate}, {"dw", dw}, {"db", db}, {"dpost_w", dpost_w}, {"dpost_b", dpost_b}, {"dgate", dgate}}, p))
        return rc;
    const bool sums = dw || db || dpost_w || dpost_b || dgate;
    if (sums && (!workspace || !aligned_to(workspace, 16) || (int64_t)workspace_bytes < skrull_residual_workspace(p)))
        return refuse("residual: workspace is null, misaligned or below %lld bytes", (long long)skrull_residual_workspace(p));
    if (p->rows > 0) {
        const Rows in_r = {"r", r, p->r_stride, p->residual_type}, in_z = {"z", z, p->z_stride, p->type};
        const Rows in_dr = {"d_r_out", d_r_out, p->d_r_out_stride, p->residual_type}, in_dy = {"dy", dy, p->dy_stride, p->type};
        const Rows out_dr = {"dr", dr, p->dr_stride, p->residual_type}, out_dz = {"dz", dz, p->dz_stride, p->type};
        for (const Rows *t : {&in_r, &in_z, &in_dr, &in_dy, &out_dr, &out_dz})
            if (t->at || (t != &in_dr && t != &in_dy))
                if (int rc = check_rows(*t, p)) return rc;
        if (!w) return refuse("residual: w is null");
        if (!stats || !aligned_to(stats, 4)) return refuse("residual: stats is null or misaligned");
        for (const Rows *out : {&out_dr, &out_dz})
            for (const Rows *in : {&in_r, &in_z, &in_dr, &in_dy})
                if (int rc = check_apart(*out, *in, p)) return rc;
        if (int rc = check_apart(out_dr, out_dz, p)) return rc;
    }
    int compute_units = 0;
    if (int rc = current_device(&compute_units)) return rc;
    hipStream_t st = (hipStream_t)hip_stream;
    hipError_t e = hipSuccess;
    int blocks = 0;
    if (p->rows > 0) {
        ResidualArgs a = args_of(p, r, z, w, post_w, post_b, gate);
        a.d_r_out = d_r_out; a.dy = dy; a.r_out = dr; a.y = dz;
        a.stats = const_cast<float *>(stats);
        a.partial = sums ? (float *)workspace : nullptr;
        a.d_r_out_stride = p->d_r_out_stride; a.dy_stride = p->dy_stride; a.r_out_stride = p->dr_stride; a.y_stride = p->dz_stride;
        blocks = (int)blocks_of(p, 2);
        launch(true, p, a, blocks, st);
        e = hipGetLastError();
    }
    if (e == hipSuccess && sums) {
        const SumsArgs a = {(const float *)workspace, post_w, post_b, gate, dw, db, dpost_w, dpost_b, dgate, blocks, p->cols, p->weight_type, p->kind == SKRULL_NORM_LAYER};
        residual_sums_kernel<<<dim3((unsigned)((p->cols + 63) / 64), 2), 1024, 0, st>>>(a);
        e = hipGetLastError();
    }
    return e == hipSuccess ? SKRULL_OK : launch_failed(e, "residual launch");
}

}  // extern "C"
