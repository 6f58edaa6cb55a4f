// Rows in registers: what the kernels of norm.hip and residual.hip share.  A row of bf16 or fp32 lies in the registers of the 64 or more lanes that
// share it, in pieces of 8 columns, from its load to its store.
#pragma once

#include <hip/hip_runtime.h>

#include "mfma.h"
#include "skrull_norm.h"

namespace {

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

inline int size_of(int type) { return type == SKRULL_TYPE_BF16 ? 2 : 4; }

}  // namespace
