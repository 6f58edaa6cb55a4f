// The norm of packed rows, forward and backward (include/skrull_norm.h).
//
// What bounds it: memory.  The forward reads x and writes y, the backward reads x and dy and writes dx, each once: a row stays in the
// registers of the lanes that share it from its load to its store, so the sums cost no second read.  Lanes keep the same columns for
// all rows of their workgroup, so w is read once per workgroup, and dw and db are summed over the rows in registers; what the workgroups
// have is added up by a second kernel in a fixed order (no atomics).  13,312 rows of 3,584 bf16 take 38 us forward (5.0 TB/s) and 60 backward with the sums
// (4.8), from memory and not from the caches; a large copy reaches 5.1.
//
// A row belongs to 64 lanes (up to 1,024 columns), 256 (up to 4,096) or 1,024 (up to 8,192), each with one or two pieces of 8 columns: so a row's
// values, weights and gradients fit the registers at every width.  (1,024 lanes of two pieces, for 16,384 columns, do not: the backward spilled.)
#include <hip/hip_runtime.h>

#include <math.h>

#include "mfma.h"
#include "ops.h"
#include "skrull_norm.h"

namespace {

struct NormArgs {
    const void *x, *w, *b, *dy;
    void *y;                 // y, or dx
    float *mean, *rstd;
    float *partial;          // [workgroups][dw, then db: cols each], or null
    int64_t x_stride, y_stride, dy_stride;
    int64_t rows;
    int32_t cols, weight_type;
    float eps, inv_cols;
};

__device__ __forceinline__ uint16_t to_bf16(float f) { return (uint16_t)pack_bf16(f, f); }

struct Bf16 {
    typedef uint16_t type;
    static __device__ __forceinline__ uint16_t put(float f) { return to_bf16(f); }
    struct Raw { uint4 v; };   // 8 values as they lie in memory
    static __device__ __forceinline__ Raw load8(const uint16_t *p)
    {
        Raw r;
        __builtin_memcpy(&r, p, sizeof r);
        return r;
    }
    static __device__ __forceinline__ Raw load_some(const uint16_t *p, int n)
    {
        uint32_t e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = i < n ? p[i] : 0;
        return Raw{make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16)};
    }
    static __device__ __forceinline__ void widen(const Raw &r, float f[8])
    {
        const uint32_t w[4] = {r.v.x, r.v.y, r.v.z, r.v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __builtin_bit_cast(float, w[i] << 16);
            f[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ void store8(uint16_t *p, const float f[8])
    {
        const uint4 v = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
        __builtin_memcpy(p, &v, sizeof v);
    }
};
struct Fp32 {
    typedef float type;
    static __device__ __forceinline__ float put(float f) { return f; }
    struct Raw { float4 a, b; };
    static __device__ __forceinline__ Raw load8(const float *p)
    {
        Raw r;
        __builtin_memcpy(&r, p, sizeof r);
        return r;
    }
    static __device__ __forceinline__ Raw load_some(const float *p, int n)
    {
        float e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = i < n ? p[i] : 0.0f;
        return Raw{make_float4(e[0], e[1], e[2], e[3]), make_float4(e[4], e[5], e[6], e[7])};
    }
    static __device__ __forceinline__ void widen(const Raw &r, float f[8])
    {
        f[0] = r.a.x; f[1] = r.a.y; f[2] = r.a.z; f[3] = r.a.w; f[4] = r.b.x; f[5] = r.b.y; f[6] = r.b.z; f[7] = r.b.w;
    }
    static __device__ __forceinline__ void store8(float *p, const float f[8])
    {
        __builtin_memcpy(p, f, 32);
    }
};

// A lane's piece of 8 columns.  The last piece of a row whose width is no multiple of 8 is its last 8 columns, of which the first ones
// belong to the lane before; rows narrower than 8 (SMALL) have one piece that is loaded value by value.  Rows need no alignment but their type's: the hardware takes 16 bytes
// from any address (7,013 rows of 1,001 bf16, backward: 34 us with a load for each value, the lanes' side by side, 17 this way).
template <bool SMALL>
struct Columns {
    int first, skip;   // the piece's values from `skip` on are this lane's (8: none); SMALL: those below 8 - skip
    __device__ __forceinline__ void init(int c, int lane, int lanes, int cols)
    {
        first = (c * lanes + lane) * 8;
        skip = max(0, min(8, first + 8 - cols));
        if (!SMALL && skip < 8) first -= skip;
    }
    __device__ __forceinline__ bool has(int i) const { return SMALL ? i < 8 - skip : i >= skip; }
};

// A lane's pieces of a row, zero where they are not its own.  They are fetched a row ahead of their use, so that they arrive while the row before is
// summed up (backward of 32,768 rows of 4,096 fp32: 313 us without, 285 with; of 8,192 of 8,192 bf16 82 and 77; 13,312 of 3,584 bf16 61 and 60, and there the
// forward 37 and 38).
template <class T, int C, bool SMALL>
struct RowPieces {
    typename T::Raw raw[C];
    __device__ __forceinline__ void init()
    {
#pragma unroll
        for (int c = 0; c < C; ++c) raw[c] = typename T::Raw{};
    }
    __device__ __forceinline__ void fetch(const typename T::type *row, const Columns<SMALL> col[C])
    {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if constexpr (SMALL) raw[c] = T::load_some(row + col[c].first, 8 - col[c].skip);
            else if (col[c].skip < 8) raw[c] = T::load8(row + col[c].first);
        }
    }
    __device__ __forceinline__ void get(const Columns<SMALL> col[C], float f[C][8]) const
    {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            T::widen(raw[c], f[c]);
            if constexpr (!SMALL) {
#pragma unroll
                for (int i = 0; i < 7; ++i) f[c][i] = col[c].has(i) ? f[c][i] : 0.0f;   // (the eighth is, or was never loaded)
            }
        }
    }
};
template <class T, bool SMALL>
__device__ __forceinline__ void store_piece(typename T::type *row, const Columns<SMALL> &k, const float f[8])
{
    if (k.skip == 0) {
        T::store8(row + k.first, f);
    } else if (k.skip < 8) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (k.has(i)) row[k.first + i] = T::put(f[i]);
        asm volatile("");   // (else the last one becomes a store of both branches, and the wide one is cut up for it)
    }
}
// The same piece of w (or b).
template <class W, bool SMALL>
__device__ __forceinline__ void load_weight(const void *w, const Columns<SMALL> &k, float f[8])
{
    typename W::Raw raw = {};
    if constexpr (SMALL) raw = W::load_some((const typename W::type *)w + k.first, 8 - k.skip);
    else if (k.skip < 8) raw = W::load8((const typename W::type *)w + k.first);
    W::widen(raw, f);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = k.has(i) ? f[i] : 0.0f;
}
template <bool SMALL>
__device__ __forceinline__ void load_weight(const void *w, int type, const Columns<SMALL> &k, float f[8])
{
    if (type == SKRULL_TYPE_BF16) load_weight<Bf16>(w, k, f);
    else load_weight<Fp32>(w, k, f);
}

// Sums of N values over the lanes of a row, in every lane.  `lds`: room for 2 x WAVES x N floats, used by turns.
template <int WAVES, int N>
__device__ __forceinline__ void row_sums(float v[N], float *lds, int &turn)
{
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int m = 32; m >= 1; m >>= 1) v[i] += __shfl_xor(v[i], m);
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

template <class T, int WAVES, int C, bool CENTER, bool SMALL>
__global__ __launch_bounds__(WAVES == 16 ? 1024 : 256) void norm_fwd_kernel(const NormArgs a)
{
    constexpr int ROWS = WAVES == 1 ? 4 : 1;   // rows of a workgroup at a time
    __shared__ float lds[2 * WAVES];
    int turn = 0;
    const int slot = ROWS > 1 ? threadIdx.x >> 6 : 0, lane = ROWS > 1 ? threadIdx.x & 63 : threadIdx.x;
    float w[C][8], b[C][8];
    Columns<SMALL> col[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        col[c].init(c, lane, 64 * WAVES, a.cols);
        load_weight(a.w, a.weight_type, col[c], w[c]);
#pragma unroll
        for (int i = 0; i < 8; ++i) b[c][i] = 0.0f;
        if (a.b) load_weight(a.b, a.weight_type, col[c], b[c]);
    }
    const typename T::type *X = (const typename T::type *)a.x;
    const int64_t stride = (int64_t)gridDim.x * ROWS;
    int64_t row = (int64_t)blockIdx.x * ROWS + slot;   // (a wavefront to a row, or all of them: no wavefront waits for one that has left)
    RowPieces<T, C, SMALL> next;
    next.init();
    if (row < a.rows) next.fetch(X + row * a.x_stride, col);
    for (; row < a.rows; row += stride) {
        float x[C][8];
        next.get(col, x);
        if (row + stride < a.rows) next.fetch(X + (row + stride) * a.x_stride, col);
        float mean = 0.0f;
        if constexpr (CENTER) {
            float s[1] = {0.0f};
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) s[0] += x[c][i];
            row_sums<WAVES, 1>(s, lds, turn);
            mean = s[0] * a.inv_cols;
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) x[c][i] = col[c].has(i) ? x[c][i] - mean : 0.0f;
        }
        float q[1] = {0.0f};
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) q[0] += x[c][i] * x[c][i];
        row_sums<WAVES, 1>(q, lds, turn);
        const float rstd = 1.0f / sqrtf(q[0] * a.inv_cols + a.eps);
        if (lane == 0) {
            if (CENTER && a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
        typename T::type *yr = (typename T::type *)a.y + row * a.y_stride;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            float y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = x[c][i] * rstd * w[c][i] + b[c][i];
            store_piece<T, SMALL>(yr, col[c], y);
        }
    }
}

template <class T, int WAVES, int C, bool CENTER, bool SMALL>
__global__ __launch_bounds__(WAVES == 16 ? 1024 : 256) void norm_bwd_kernel(const NormArgs a)
{
    constexpr int ROWS = WAVES == 1 ? 4 : 1;
    __shared__ float lds[2 * WAVES * 2];
    int turn = 0;
    const int slot = ROWS > 1 ? threadIdx.x >> 6 : 0, lane = ROWS > 1 ? threadIdx.x & 63 : threadIdx.x;
    float w[C][8], dw[C][8], db[C][8];
    Columns<SMALL> col[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        col[c].init(c, lane, 64 * WAVES, a.cols);
        load_weight(a.w, a.weight_type, col[c], w[c]);
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[c][i] = db[c][i] = 0.0f;
    }
    const typename T::type *X = (const typename T::type *)a.x, *DY = (const typename T::type *)a.dy;
    const int64_t stride = (int64_t)gridDim.x * ROWS;
    int64_t row = (int64_t)blockIdx.x * ROWS + slot;
    RowPieces<T, C, SMALL> next_x, next_dy;
    next_x.init();
    next_dy.init();
    float next_mean = 0.0f, next_rstd = 0.0f;
    auto fetch = [&](int64_t r) {
        next_x.fetch(X + r * a.x_stride, col);
        next_dy.fetch(DY + r * a.dy_stride, col);
        if (CENTER) next_mean = a.mean[r];
        next_rstd = a.rstd[r];
    };
    if (row < a.rows) fetch(row);
    for (; row < a.rows; row += stride) {
        const float mean = next_mean, rstd = next_rstd;
        float h[C][8], g[C][8];
        next_x.get(col, h);
        next_dy.get(col, g);
        if (row + stride < a.rows) fetch(row + stride);
        float s[2] = {0.0f, 0.0f};   // sum g h, sum g
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                h[c][i] = (h[c][i] - mean) * rstd;
                dw[c][i] += g[c][i] * h[c][i];
                if (CENTER) db[c][i] += g[c][i];
                g[c][i] *= w[c][i];   // (zero behind the last column, whatever h is there)
                s[0] += g[c][i] * h[c][i];
                if (CENTER) s[1] += g[c][i];
            }
        if constexpr (CENTER) row_sums<WAVES, 2>(s, lds, turn);
        else row_sums<WAVES, 1>(s, lds, turn);
        const float m0 = s[0] * a.inv_cols, m1 = CENTER ? s[1] * a.inv_cols : 0.0f;
        typename T::type *out = (typename T::type *)a.y + row * a.y_stride;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            float dx[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) dx[i] = (g[c][i] - m1 - h[c][i] * m0) * rstd;
            store_piece<T, SMALL>(out, col[c], dx);
        }
    }
    if (!a.partial) return;
    float *line = a.partial + (int64_t)blockIdx.x * 2 * a.cols;
    if constexpr (ROWS == 1) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            store_piece<Fp32, SMALL>(line, col[c], dw[c]);
            if (CENTER) store_piece<Fp32, SMALL>(line + a.cols, col[c], db[c]);
        }
    } else {   // the wavefronts' own sums first
        __shared__ float sums[ROWS][C * 8][64];
#pragma unroll
        for (int which = 0; which < (CENTER ? 2 : 1); ++which) {
            if (which) __syncthreads();
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) sums[slot][c * 8 + i][lane] = which ? db[c][i] : dw[c][i];
            __syncthreads();
            if (slot == 0) {
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    float f[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[i] = (sums[0][c * 8 + i][lane] + sums[1][c * 8 + i][lane]) + (sums[2][c * 8 + i][lane] + sums[3][c * 8 + i][lane]);
                    store_piece<Fp32, SMALL>(line + which * a.cols, col[c], f);
                }
            }
        }
    }
}

// dw and db from the partial sums: 64 columns to a workgroup, 16 wavefronts share the lines, in the order of their number.
__global__ __launch_bounds__(1024) void norm_sums_kernel(const float *partial, int lines, int cols, void *dw, void *db, int weight_type)
{
    __shared__ float part[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
    void *out = blockIdx.y ? db : dw;
    if (!out) return;   // (the whole workgroup)
    float s = 0.0f;
    if (c < cols) {
        const float *p = partial + blockIdx.y * (int64_t)cols + c;
#pragma unroll 8
        for (int i = wave; i < lines; i += 16) s += p[(int64_t)i * 2 * cols];
    }
    part[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && c < cols) {
        s = 0.0f;
#pragma unroll
        for (int k = 0; k < 16; ++k) s += part[k][lane];
        if (weight_type == SKRULL_TYPE_BF16) ((uint16_t *)out)[c] = to_bf16(s);
        else ((float *)out)[c] = s;
    }
}

int size_of(int type) { return type == SKRULL_TYPE_BF16 ? 2 : 4; }

int check(const skrull_norm_t *p)
{
    if (!p) return refuse("norm: null pointer");
    if (p->rows < 0 || p->rows > INT32_MAX) return refuse("norm: %lld rows", (long long)p->rows);
    if (p->cols < 1 || p->cols > SKRULL_NORM_MAX_COLS) return refuse("norm: %d columns, at most %d", p->cols, SKRULL_NORM_MAX_COLS);
    if (p->kind != SKRULL_NORM_RMS && p->kind != SKRULL_NORM_LAYER) return refuse("norm: unknown kind %d", p->kind);
    if (p->type != SKRULL_TYPE_BF16 && p->type != SKRULL_TYPE_FP32) return refuse("norm: unknown type %d", p->type);
    if (p->weight_type != SKRULL_TYPE_BF16 && p->weight_type != SKRULL_TYPE_FP32) return refuse("norm: unknown weight_type %d", p->weight_type);
    if (!isfinite(p->eps) || !(p->eps >= 0.0f)) return refuse("norm: eps must be finite and not negative");
    return SKRULL_OK;
}

int check_rows(const char *name, const void *ptr, int64_t stride, const skrull_norm_t *p)
{
    if (!ptr || !aligned_to(ptr, size_of(p->type))) return refuse("norm: %s is null or misaligned", name);
    if (stride < p->cols || stride > INT64_MAX / 8 / (p->rows + 1)) return refuse("norm: stride of %s", name);
    return SKRULL_OK;
}
int check_weight(const char *name, const void *ptr, const skrull_norm_t *p)
{
    if (ptr && !aligned_to(ptr, size_of(p->weight_type))) return refuse("norm: %s is misaligned", name);
    return SKRULL_OK;
}
int check_apart(const char *out_name, const void *out, int64_t out_stride, const char *in_name, const void *in, int64_t in_stride, const skrull_norm_t *p)
{
    if (p->rows == 0 || (in == out && in_stride == out_stride)) return SKRULL_OK;
    const int64_t s = size_of(p->type);
    if (overlap(in, ((p->rows - 1) * in_stride + p->cols) * s, out, ((p->rows - 1) * out_stride + p->cols) * s))
        return refuse("norm: %s overlaps %s", out_name, in_name);
    return SKRULL_OK;
}

int waves_of(int cols) { return cols <= 1024 ? 1 : cols <= 4096 ? 4 : 16; }

// Workgroups of the backward, each with a line of partial sums: as many as have 32 KB of rows among them on a compute unit, one to four (13,312 x 3,584 bf16:
// 60 us with two, 64 with one or four; 32,768 x 4,096 fp32: 285 with one, 311 with two or four; 26,624 x 896 bf16: 33 with two, 36 with one, 40 with four).
constexpr int kComputeUnits = 256;
int64_t bwd_blocks(const skrull_norm_t *p)
{
    const int waves = waves_of(p->cols), rows = waves == 1 ? 4 : 1;
    const int64_t row_bytes = (int64_t)rows * p->cols * size_of(p->type) * 2, fit = 32768 / row_bytes;
    const int64_t most = (fit < 1 ? 1 : fit > 4 ? 4 : fit) * kComputeUnits, need = (p->rows + rows - 1) / rows;
    return need < most ? need : most;
}

template <class T, bool CENTER>
void launch(bool backward, const NormArgs &a, int blocks, hipStream_t st)
{
    const int cols = a.cols;
#define SKRULL_NORM_CASE(WAVES, C, SMALL)                                                                                                     \
    do {                                                                                                                               \
        if (backward) norm_bwd_kernel<T, WAVES, C, CENTER, SMALL><<<blocks, WAVES == 16 ? 1024 : 256, 0, st>>>(a);                     \
        else norm_fwd_kernel<T, WAVES, C, CENTER, SMALL><<<blocks, WAVES == 16 ? 1024 : 256, 0, st>>>(a);                                     \
    } while (0)
    if (cols < 8) SKRULL_NORM_CASE(1, 1, true);
    else if (cols <= 512) SKRULL_NORM_CASE(1, 1, false);
    else if (cols <= 1024) SKRULL_NORM_CASE(1, 2, false);
    else if (cols <= 2048) SKRULL_NORM_CASE(4, 1, false);
    else if (cols <= 4096) SKRULL_NORM_CASE(4, 2, false);
    else SKRULL_NORM_CASE(16, 1, false);
#undef SKRULL_NORM_CASE
}
void launch(bool backward, const skrull_norm_t *p, const NormArgs &a, int blocks, hipStream_t st)
{
    if (p->type == SKRULL_TYPE_BF16) {
        if (p->kind == SKRULL_NORM_LAYER) launch<Bf16, true>(backward, a, blocks, st);
        else launch<Bf16, false>(backward, a, blocks, st);
    } else {
        if (p->kind == SKRULL_NORM_LAYER) launch<Fp32, true>(backward, a, blocks, st);
        else launch<Fp32, false>(backward, a, blocks, st);
    }
}

}  // namespace

extern "C" {

int skrull_norm_fwd(const skrull_norm_t *p, const void *x, const void *w, const void *b, void *y, float *mean, float *rstd, void *hip_stream)
{
    if (int rc = check(p)) return rc;
    if (p->rows == 0) return SKRULL_OK;
    if (int rc = check_rows("x", x, p->x_stride, p)) return rc;
    if (int rc = check_rows("y", y, p->y_stride, p)) return rc;
    if (!w) return refuse("norm: w is null");
    if (int rc = check_weight("w", w, p)) return rc;
    if (int rc = check_weight("b", b, p)) return rc;
    if (b && p->kind == SKRULL_NORM_RMS) return refuse("norm: no bias without a mean (SKRULL_NORM_RMS)");
    if (!aligned_to(mean, 4) || !aligned_to(rstd, 4)) return refuse("norm: mean or rstd is misaligned");
    if (int rc = check_apart("y", y, p->y_stride, "x", x, p->x_stride, p)) return rc;
    int compute_units = 0;
    if (int rc = current_device(&compute_units)) return rc;
    NormArgs a = {};
    a.x = x; a.w = w; a.b = b; a.y = y; a.mean = mean; a.rstd = rstd;
    a.x_stride = p->x_stride; a.y_stride = p->y_stride; a.rows = p->rows; a.cols = p->cols; a.weight_type = p->weight_type;
    a.eps = p->eps; a.inv_cols = 1.0f / (float)p->cols;
    const int waves = waves_of(p->cols), rows = waves == 1 ? 4 : 1;
    // (13,312 x 3,584 bf16, layer norm: 39 us with four workgroups to a compute unit, 43 with eight; 26,624 x 896 without a mean: 19 and 20.5)
    const int64_t most = (int64_t)compute_units * (waves == 16 ? 2 : 4), need = (p->rows + rows - 1) / rows;
    launch(false, p, a, (int)(need < most ? need : most), (hipStream_t)hip_stream);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SKRULL_OK : launch_failed(e, "norm launch");
}

int64_t skrull_norm_workspace(const skrull_norm_t *p)
{
    return check(p) == SKRULL_OK ? bwd_blocks(p) * 2 * p->cols * 4 + 16 : 0;
}

int skrull_norm_bwd(const skrull_norm_t *p, const void *x, const void *w, const float *mean, const float *rstd, const void *dy,
                    void *dx, void *dw, void *db, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (int rc = check(p)) return rc;
    if (int rc = check_weight("dw", dw, p)) return rc;
    if (int rc = check_weight("db", db, p)) return rc;
    const bool sums = dw || db;
    if (db && p->kind == SKRULL_NORM_RMS) return refuse("norm: no gradient of a bias without a mean (SKRULL_NORM_RMS)");
    if (sums && (!workspace || !aligned_to(workspace, 16) || (int64_t)workspace_bytes < skrull_norm_workspace(p)))
        return refuse("norm: workspace is null, misaligned or below %lld bytes", (long long)skrull_norm_workspace(p));
    if (p->rows > 0) {
        if (int rc = check_rows("x", x, p->x_stride, p)) return rc;
        if (int rc = check_rows("dy", dy, p->dy_stride, p)) return rc;
        if (int rc = check_rows("dx", dx, p->dx_stride, p)) return rc;
        if (!w) return refuse("norm: w is null");
        if (int rc = check_weight("w", w, p)) return rc;
        if (!rstd || !aligned_to(rstd, 4) || (p->kind == SKRULL_NORM_LAYER && (!mean || !aligned_to(mean, 4))))
            return refuse("norm: mean or rstd is null or misaligned");
        if (int rc = check_apart("dx", dx, p->dx_stride, "x", x, p->x_stride, p)) return rc;
        if (int rc = check_apart("dx", dx, p->dx_stride, "dy", dy, p->dy_stride, p)) return rc;
    }
    int compute_units = 0;
    if (int rc = current_device(&compute_units)) return rc;
    hipStream_t st = (hipStream_t)hip_stream;
    hipError_t e = hipSuccess;
    int blocks = 0;
    if (p->rows > 0) {
        NormArgs a = {};
        a.x = x; a.w = w; a.dy = dy; a.y = dx; a.mean = const_cast<float *>(mean); a.rstd = const_cast<float *>(rstd);
        a.partial = sums ? (float *)workspace : nullptr;
        a.x_stride = p->x_stride; a.y_stride = p->dx_stride; a.dy_stride = p->dy_stride; a.rows = p->rows; a.cols = p->cols;
        a.weight_type = p->weight_type;
        a.inv_cols = 1.0f / (float)p->cols;
        blocks = (int)bwd_blocks(p);
        launch(true, p, a, blocks, st);
        e = hipGetLastError();
    }
    if (e == hipSuccess && sums) {
        norm_sums_kernel<<<dim3((unsigned)((p->cols + 63) / 64), 2), 1024, 0, st>>>((const float *)workspace, blocks, p->cols, dw, db, p->weight_type);
        e = hipGetLastError();
    }
    return e == hipSuccess ? SKRULL_OK : launch_failed(e, "norm launch");
}

}  // extern "C"
