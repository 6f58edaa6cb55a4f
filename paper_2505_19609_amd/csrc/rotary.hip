// Rotary positions of a plan's packed rows (include/skrull_rotary.h).
//
// What bounds it: every element of Q and K is read and written once, 4 bytes, and meets two products; the
// sines and cosines are one pair per (row, pair of elements), shared by all heads of the row.  So a workgroup takes a few whole rows, of Q and K
// together where both hold the same rows, asks for their heads, 16 bytes per load, forms their sines and cosines once into LDS and
// stores what it makes of both.  The positions come from the plan's descriptor (which segment a row is in), so nothing but the tensors themselves is read per element.
// 32,768 tokens, 32/8 heads of 128, out of a projection's rows: 671 MB in 118 us, 5.7 TB/s; a large copy reaches 5.1 to 5.4.
#include <math.h>

#include <hip/hip_bf16.h>

#include "mfma.h"
#include "ops.h"
#include "skrull_rotary.h"

namespace {

constexpr int kThreads = 256;
constexpr int kMaxRows = 32;    // rows of a workgroup at most
constexpr int kMaxPairs = 64;   // head_dim / 2

struct Tensor {
    const uint16_t *in;
    uint16_t *out;
    int64_t in_stride, out_stride;
    int32_t heads, head_units, row_units;   // units of a head: those that are turned, and the others where `out` is other memory
    uint64_t inv_row, inv_head;  // ceil(2^40 / units of a row, of a head)
};
// Rows that workgroups share out, and the tensors that hold them.
struct Rows {
    const int32_t *cu;      // [NS+1] first row of each segment
    const int32_t *begin;   // [NS] position of its first row, or null: 0
    int32_t rows, each, blocks, tensors;   // rows of a workgroup; workgroups; one or two tensors
    Tensor t[2];
};

struct Args {
    Rows r[2];
    int32_t NS, head_dim, rotary_dim, scaling;
    double log2_base, factor, turns_scale, low_turns, high_turns;   // turns_scale: original_length
    float amplitude, sign;
};

// x / d with inv = ceil(2^40 / d): exact while x * d < 2^40
__device__ __forceinline__ int quotient40(int x, uint64_t inv) { return (int)(((uint64_t)(uint32_t)x * inv) >> 40); }

// Turns per position of pair i.
__device__ double turns_of(const Args &a, int i)
{
    constexpr double kTurn = 0.15915494309189533577;  // 1 / (2 pi)
    const double f = exp2(-a.log2_base * (double)(2 * i) / (double)a.rotary_dim) * kTurn;
    if (a.scaling == SKRULL_ROTARY_LINEAR) return f / a.factor;
    if (a.scaling == SKRULL_ROTARY_PARTS) {
        const double g = fmin(fmax((a.turns_scale * f - a.low_turns) / (a.high_turns - a.low_turns), 0.0), 1.0);
        return f * (g + (1.0 - g) / a.factor);
    }
    return f;
}

__device__ __forceinline__ float lo_of(uint32_t u) { return __builtin_bit_cast(float, u << 16); }
__device__ __forceinline__ float hi_of(uint32_t u) { return __builtin_bit_cast(float, u & 0xffff0000u); }

// The positions of `rows` (at most 32) rows from row0 on, in the lanes of one wavefront: 64 segments' first rows are compared at a time, so
// a row's segment is two or three loads away in any micro-batch.
__device__ __forceinline__ int position_of(const Rows &w, int NS, int row0, int rows, int lane)
{
    int lo = 0, len = NS;   // row0 lies in one of the segments lo .. lo + len - 1
    while (len > 31) {
        const int step = (len + 63) / 64, i = lane * step;
        const int first = i < len ? w.cu[lo + i] : INT32_MAX;
        lo += (__popcll(__ballot(first <= row0)) - 1) * step;
        len = min(step, NS - lo);
    }
    const int first = lo + lane < NS ? w.cu[lo + lane] : INT32_MAX;   // (31 segments and one more per row are in reach)
    int segment = lo;
    for (int r = 0; r < rows; ++r) {
        const int s = lo + __popcll(__ballot(first <= row0 + r)) - 1;
        if (lane == r) segment = s;
    }
    return row0 + lane - __shfl(first, segment - lo) + (w.begin ? w.begin[segment] : 0);
}

// What a lane moves at a time: 16 bytes of a head, 4 pairs (interleaved), or two pieces of 16 bytes, 8 pairs (half; behind rotary_dim two pieces side by side).
template <bool INTERLEAVED>
struct Unit {
    static constexpr int kPieces = INTERLEAVED ? 1 : 2;
    uint16_t *out;
    int second, angle;   // elements to the second piece; the first pair's place among the angles, -1: as it is, -2: there is no such unit
    uint4 v[kPieces];
    // Unit i of the workgroup's rows, first one tensor's, then the other's; loaded.
    __device__ __forceinline__ void load(const Args &a, const Rows &w, int i, int units0, int units, int row0)
    {
        angle = -2;
        if (i >= units) return;
        const bool other = i >= units0;
        const Tensor &t = w.t[other];
        i -= other ? units0 : 0;
        const int r = quotient40(i, t.inv_row), x = i - r * t.row_units, head = quotient40(x, t.inv_head), u = x - head * t.head_units;
        const int pairs = a.rotary_dim / 2, turned = pairs / (4 * kPieces);
        const bool turns = u < turned;
        const int64_t row = row0 + r;
        const int at = head * a.head_dim + (INTERLEAVED ? u * 8 : turns ? u * 8 : a.rotary_dim + (u - turned) * 16);
        second = turns ? pairs : 8;
        angle = turns ? r * pairs + u * (4 * kPieces) : -1;
        const uint16_t *in = t.in + row * t.in_stride + at;
        out = t.out + row * t.out_stride + at;
        v[0] = *(const uint4 *)in;
        if constexpr (!INTERLEAVED) v[1] = *(const uint4 *)(in + second);
    }
    __device__ __forceinline__ void store(const float2 *turn)
    {
        if (angle == -2) return;
        if (angle >= 0) {
            const float2 *cs = turn + angle;
            if constexpr (INTERLEAVED) {
                uint32_t w[4] = {v[0].x, v[0].y, v[0].z, v[0].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float x0 = lo_of(w[j]), x1 = hi_of(w[j]), c = cs[j].x, s = cs[j].y;
                    w[j] = pack_bf16(x0 * c - x1 * s, x0 * s + x1 * c);
                }
                v[0] = make_uint4(w[0], w[1], w[2], w[3]);
            } else {
                uint32_t a0[4] = {v[0].x, v[0].y, v[0].z, v[0].w}, a1[4] = {v[1].x, v[1].y, v[1].z, v[1].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float p0 = lo_of(a0[j]), p1 = hi_of(a0[j]), q0 = lo_of(a1[j]), q1 = hi_of(a1[j]);
                    const float c0 = cs[2 * j].x, s0 = cs[2 * j].y, c1 = cs[2 * j + 1].x, s1 = cs[2 * j + 1].y;
                    a0[j] = pack_bf16(p0 * c0 - q0 * s0, p1 * c1 - q1 * s1);
                    a1[j] = pack_bf16(p0 * s0 + q0 * c0, p1 * s1 + q1 * c1);
                }
                v[0] = make_uint4(a0[0], a0[1], a0[2], a0[3]);
                v[1] = make_uint4(a1[0], a1[1], a1[2], a1[3]);
            }
        }
        *(uint4 *)out = v[0];
        if constexpr (!INTERLEAVED) *(uint4 *)(out + second) = v[1];
    }
};

template <bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void rotary_kernel(const Args a)
{
    __shared__ double freq[kMaxPairs];
    __shared__ int pos[kMaxRows];
    __shared__ float2 turn[kMaxRows * kMaxPairs];   // cos, sin
    const int which = (int)blockIdx.x >= a.r[0].blocks;
    const Rows &w = a.r[which];
    const int row0 = ((int)blockIdx.x - (which ? a.r[0].blocks : 0)) * w.each;
    const int rows = min(w.each, w.rows - row0);
    const int pairs = a.rotary_dim / 2;
    const int tid = threadIdx.x;

    // The first units are on their way while the angles are formed (26,624 tokens, 14/2 heads of 64, half of each turned: 27 us, 31 with the angles first;
    // 932 tokens, 4/4 heads: 2.9 and 3.4).
    constexpr int kUnits = INTERLEAVED ? 4 : 2;
    const int units0 = rows * w.t[0].row_units, units = units0 + rows * w.t[1].row_units;
    Unit<INTERLEAVED> unit[kUnits];
#pragma unroll
    for (int j = 0; j < kUnits; ++j) unit[j].load(a, w, tid + j * kThreads, units0, units, row0);

    if (tid < pairs) freq[tid] = turns_of(a, tid);
    if (tid >= 64 && tid < 128) {   // (another wavefront than that of the frequencies)
        const int p = position_of(w, a.NS, row0, rows, tid - 64);
        if (tid - 64 < rows) pos[tid - 64] = p;
    }
    __syncthreads();
    for (int i = tid; i < rows * pairs; i += kThreads) {
        const int r = i / pairs, p = i - r * pairs;
        const double turns = (double)pos[r] * freq[p];
        float s, c;
        sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
        turn[i] = make_float2(c * a.amplitude, s * a.amplitude * a.sign);
    }
    __syncthreads();
    for (int base = kUnits * kThreads;; base += kUnits * kThreads) {
#pragma unroll
        for (int j = 0; j < kUnits; ++j) unit[j].store(turn);
        if (base >= units) break;
#pragma unroll
        for (int j = 0; j < kUnits; ++j) unit[j].load(a, w, base + tid + j * kThreads, units0, units, row0);
    }
}

uint64_t inverse40(int d) { return ((1ull << 40) + (uint64_t)d - 1) / (uint64_t)d; }

}  // namespace

extern "C" {

int skrull_rotary_check(const skrull_rotary_t *r)
{
    if (!r) return refuse("rotary: null pointer");
    if (r->head_dim != 64 && r->head_dim != 128) return refuse("rotary: head_dim %d is not 64 or 128", r->head_dim);
    if (r->rotary_dim < 16 || r->rotary_dim > r->head_dim || r->rotary_dim % 16 != 0)
        return refuse("rotary: rotary_dim %d is not a multiple of 16 from 16 to head_dim", r->rotary_dim);
    if (r->layout != SKRULL_ROTARY_HALF && r->layout != SKRULL_ROTARY_INTERLEAVED) return refuse("rotary: unknown layout %d", r->layout);
    if (r->scaling < SKRULL_ROTARY_PLAIN || r->scaling > SKRULL_ROTARY_PARTS) return refuse("rotary: unknown scaling %d", r->scaling);
    if (!isfinite(r->base) || !(r->base > 1.0)) return refuse("rotary: base must be finite and above 1");
    if (!isfinite(r->factor) || !(r->factor >= 1.0)) return refuse("rotary: factor must be finite and at least 1");
    if (r->scaling == SKRULL_ROTARY_PLAIN && r->factor != 1.0) return refuse("rotary: a factor needs a scaling");
    if (!isfinite(r->amplitude) || !(r->amplitude > 0.0)) return refuse("rotary: amplitude must be finite and positive");
    if (r->scaling == SKRULL_ROTARY_PARTS) {
        if (!isfinite(r->original_length) || !(r->original_length > 0.0)) return refuse("rotary: original_length must be finite and positive");
        if (!isfinite(r->low_turns) || !isfinite(r->high_turns) || !(r->low_turns >= 0.0) || !(r->low_turns < r->high_turns))
            return refuse("rotary: low_turns and high_turns must be finite, 0 <= low_turns < high_turns");
    }
    return SKRULL_OK;
}

int skrull_rotary(const skrull_attn_plan_t *plan, const skrull_rotary_t *r, const skrull_rotary_tensor_t *first,
                  const skrull_rotary_tensor_t *second, int inverse, void *hip_stream)
{
    if (!plan || !first) return refuse("rotary: null pointer");
    if (int rc = skrull_rotary_check(r)) return rc;
    if (r->head_dim != plan->d) return refuse("rotary: head_dim %d, the plan's is %d", r->head_dim, plan->d);
    Args a = {};
    a.NS = plan->NS;
    a.head_dim = r->head_dim;
    a.rotary_dim = r->rotary_dim;
    a.scaling = r->scaling;
    a.log2_base = log2(r->base);
    if (r->scaling == SKRULL_ROTARY_NTK)
        a.log2_base += log2(r->factor) * (double)r->rotary_dim / (double)(r->rotary_dim - 2);
    a.factor = r->factor;
    a.turns_scale = r->original_length;
    a.low_turns = r->low_turns;
    a.high_turns = r->high_turns;
    a.amplitude = (float)r->amplitude;
    a.sign = inverse ? -1.0f : 1.0f;
    const skrull_rotary_tensor_t *given[2] = {first, second};
    int64_t blocks = 0;
    int groups = 0;
    for (int i = 0; i < 2; ++i) {
        const skrull_rotary_tensor_t *g = given[i];
        if (!g) continue;
        if (!g->in || !g->out || !aligned_to(g->in, 16) || !aligned_to(g->out, 16)) return refuse("rotary: tensor %d is null or not 16-byte aligned", i);
        if (g->heads < 1 || g->heads > 4096) return refuse("rotary: tensor %d has %d heads", i, g->heads);
        if (g->rows != SKRULL_ROWS_Q && g->rows != SKRULL_ROWS_K) return refuse("rotary: tensor %d is of unknown rows %d", i, g->rows);
        const int64_t width = (int64_t)g->heads * r->head_dim;
        if (g->in_stride < width || g->out_stride < width || g->in_stride % 8 != 0 || g->out_stride % 8 != 0)
            return refuse("rotary: strides of tensor %d must be multiples of 8 and at least heads * head_dim", i);
        // (sequences that are whole have the same rows in both packings; any other has more keys than queries)
        const bool q_rows = g->rows == SKRULL_ROWS_Q || plan->total_q == plan->total_k;
        const int64_t n = q_rows ? plan->total_q : plan->total_k;
        if (g->in_stride > INT64_MAX / 4 / n || g->out_stride > INT64_MAX / 4 / n) return refuse("rotary: stride of tensor %d", i);
        const int64_t in_bytes = ((n - 1) * g->in_stride + width) * 2, out_bytes = ((n - 1) * g->out_stride + width) * 2;
        const bool in_place = g->in == g->out && g->in_stride == g->out_stride;
        if (!in_place && overlap(g->in, in_bytes, g->out, out_bytes)) return refuse("rotary: out of tensor %d overlaps its in", i);
        const int32_t *cu = q_rows ? plan->cu_q : plan->cu_k;
        Rows &w = groups > 0 && a.r[0].cu == cu ? a.r[0] : a.r[groups++];
        w.cu = cu;
        w.begin = q_rows ? plan->q_begin : nullptr;
        w.rows = (int32_t)n;
        Tensor &t = w.t[w.tensors++];
        t.in = (const uint16_t *)g->in;
        t.out = (uint16_t *)g->out;
        t.in_stride = g->in_stride;
        t.out_stride = g->out_stride;
        t.heads = g->heads;
        t.head_units = (in_place ? r->rotary_dim : r->head_dim) / (r->layout == SKRULL_ROTARY_INTERLEAVED ? 8 : 16);
        t.row_units = t.head_units * g->heads;
        t.inv_head = inverse40(t.head_units);
        t.inv_row = inverse40(t.row_units);
    }
    for (int i = 0; i < groups; ++i) {
        Rows &w = a.r[i];
        // up to 16 KB in a workgroup's rows (32,768 tokens, 32/8 heads of 128: 117 us, 123 with 32 KB), fewer where that makes less than 512 of them
        // (3,991 tokens, 14/2 heads of 64, the angles first: 5.8 us; 6.2 without this, 8.5 with single rows)
        const int64_t width = (int64_t)(w.t[0].heads + w.t[1].heads) * r->head_dim;
        int32_t each = kMaxRows;
        while (each > 1 && (each * width > 8192 || (int64_t)w.rows < each * 512)) each /= 2;
        w.each = each;
        w.blocks = (w.rows + each - 1) / each;
        blocks += w.blocks;
    }
    if (int rc = plan_on_current_device(plan)) return rc;
    if (blocks > INT32_MAX) return refuse("rotary: too many rows");
    if (r->layout == SKRULL_ROTARY_INTERLEAVED) rotary_kernel<true><<<(int)blocks, kThreads, 0, (hipStream_t)hip_stream>>>(a);
    else rotary_kernel<false><<<(int)blocks, kThreads, 0, (hipStream_t)hip_stream>>>(a);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SKRULL_OK : launch_failed(e, "rotary launch");
}

}  // extern "C"
