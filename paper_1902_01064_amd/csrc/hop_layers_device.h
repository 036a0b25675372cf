// Device code that the kernels of hop_product.hip and hop_residual.hip share.
#pragma once

#include <hip/hip_runtime.h>

#include "hop_layers_internal.h"

namespace hopl {

typedef __bf16 bf16;
typedef bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// Global memory takes 128-bit accesses at any address, so rows need no alignment beyond an element's.
typedef bf16x8 bf16x8_any __attribute__((aligned(2)));
typedef bf16x4 bf16x4_any __attribute__((aligned(2)));
typedef f32x8 f32x8_any __attribute__((aligned(4)));
typedef f32x4 f32x4_any __attribute__((aligned(4)));

// Pointers out of structures are generic to the compiler; all of them are global memory (flat accesses would also count on the
// LDS counter).
#define HOPL_GLOBAL __attribute__((address_space(1)))

// The first n (1 <= n) of a vector's elements from p on, the rest zero: as many loads as the vector is long whatever n is, all at once -
// behind branches each would wait for the one before.
template <typename V, typename T>
__device__ __forceinline__ V load_short(const T* p, int n) {
    constexpr int kN = sizeof(V) / sizeof(T);
    V v;
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] = ((const HOPL_GLOBAL T*)p)[i < n ? i : 0];
#pragma unroll
    for (int i = 1; i < kN; ++i) v[i] = i < n ? v[i] : (T)0.f;
    return v;
}
// Eight consecutive elements from p on, as floats; the first n of them exist (n >= 8: all).
__device__ __forceinline__ f32x8 load8(const float* p, int n) {
    if (n >= 8) return *(const HOPL_GLOBAL f32x8_any*)p;
    return load_short<f32x8>(p, n);
}
__device__ __forceinline__ void store8(float* p, int n, f32x8 v) {
    if (n >= 8) {
        *(HOPL_GLOBAL f32x8_any*)p = v;
        return;
    }
#pragma unroll
    for (int i = 0; i < 7; ++i)
        if (i < n) ((HOPL_GLOBAL float*)p)[i] = v[i];
}
__device__ __forceinline__ void store8(bf16* p, int n, f32x8 v) {
    const bf16x8 r = __builtin_convertvector(v, bf16x8);      // to nearest, ties to even
    if (n >= 8) {
        *(HOPL_GLOBAL bf16x8_any*)p = r;
        return;
    }
#pragma unroll
    for (int i = 0; i < 7; ++i)
        if (i < n) ((HOPL_GLOBAL bf16*)p)[i] = r[i];
}

__device__ __forceinline__ int clamp_int(int v, int lo, int hi) { return v < lo ? lo : v > hi ? hi : v; }

// Rows of a launch are handed out in pieces of 1 << shift rows of one group; piece number `piece` -> its group and rows
// [*r0, *r1).  False: there are fewer pieces.  The host cannot know how many there are, since the table is on the device, and
// launches rows / step + G of them at most.  Every wavefront works it out for itself: 64 groups at a time, a scan of their
// pieces and a ballot, one load deep.  Whatever the table holds, 0 <= *r0 < *r1 <= rows.
__device__ __forceinline__ bool find_piece(const HopRows& rows, int shift, int piece, int* g, int* r0, int* r1) {
    const int step = 1 << shift;
    if (!rows.begin) {
        *g = 0;
        const int64_t at = (int64_t)piece << shift;
        if (at >= rows.rows) return false;
        *r0 = (int)at;
        *r1 = rows.rows - (int)at < step ? rows.rows : (int)at + step;
        return true;
    }
    const int lane = threadIdx.x & 63;
    const HOPL_GLOBAL int32_t* table = (const HOPL_GLOBAL int32_t*)rows.begin;
    int seen = 0;
    for (int base = 0; base < rows.G; base += 64) {
        const int mine = base + lane;
        int b = 0, e = 0;
        if (mine < rows.G) {
            b = clamp_int(table[mine], 0, rows.rows);
            e = clamp_int(table[mine + 1], b, rows.rows);
        }
        int scan = (int)(((int64_t)(e - b) + step - 1) >> shift);
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int before = __shfl_up(scan, o);
            if (lane >= o) scan += before;
        }
        const uint64_t behind = __ballot(seen + scan > piece);
        if (behind) {
            const int l = __builtin_ctzll(behind);
            const int gb = __builtin_amdgcn_readlane(b, l), ge = __builtin_amdgcn_readlane(e, l);
            const int first = seen + __builtin_amdgcn_readlane(scan, l) - (int)(((int64_t)(ge - gb) + step - 1) >> shift);
            const int64_t at = gb + ((int64_t)(piece - first) << shift);
            if (at < gb || at >= ge) return false;        // only where a broken table made the sums overflow
            *g = base + l;
            *r0 = (int)at;
            *r1 = ge - at < step ? ge : (int)at + step;
            return true;
        }
        seen += __builtin_amdgcn_readlane(scan, 63);
    }
    return false;
}

// How many pieces of 1 << shift rows there are.
__device__ __forceinline__ int count_pieces(const HopRows& rows, int shift) {
    const int step = 1 << shift;
    if (!rows.begin) return (int)(((int64_t)rows.rows + step - 1) >> shift);
    const HOPL_GLOBAL int32_t* table = (const HOPL_GLOBAL int32_t*)rows.begin;
    int n = 0;
    for (int g = threadIdx.x & 63; g < rows.G; g += 64) {
        const int b = clamp_int(table[g], 0, rows.rows), e = clamp_int(table[g + 1], b, rows.rows);
        n += (int)(((int64_t)(e - b) + step - 1) >> shift);
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) n += __shfl_xor(n, o);
    return __builtin_amdgcn_readfirstlane(n);
}

// The same with the shorter pieces at the groups' ends spread evenly between the whole ones: the short ones are bound by reading weights, the
// whole ones by arithmetic, and they are to run side by side.  count_whole gives both numbers; find_whole takes a piece by its place.
struct WholePieces {
    int whole, rest;
};
__device__ __forceinline__ WholePieces count_whole(const HopRows& rows, int shift) {
    const int part = (1 << shift) - 1;
    if (!rows.begin) return {rows.rows >> shift, (rows.rows & part) != 0};
    const HOPL_GLOBAL int32_t* table = (const HOPL_GLOBAL int32_t*)rows.begin;
    int whole = 0, rest = 0;
    for (int g = threadIdx.x & 63; g < rows.G; g += 64) {
        const int b = clamp_int(table[g], 0, rows.rows), n = clamp_int(table[g + 1], b, rows.rows) - b;
        whole += n >> shift;
        rest += (n & part) != 0;
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) {
        whole += __shfl_xor(whole, o);
        rest += __shfl_xor(rest, o);
    }
    return {__builtin_amdgcn_readfirstlane(whole), __builtin_amdgcn_readfirstlane(rest)};
}
__device__ __forceinline__ bool find_whole(const HopRows& rows, int shift, WholePieces all, int piece, int* g, int* r0, int* r1) {
    const int step = 1 << shift;
    if (!rows.begin) {
        *g = 0;
        *r0 = piece << shift;
        *r1 = min(*r0 + step, rows.rows);
        return *r0 < *r1;
    }
    const int64_t total = (int64_t)all.whole + all.rest;
    const int rests = (int)(((int64_t)piece * all.rest) / total), then = (int)(((int64_t)(piece + 1) * all.rest) / total);
    const bool last = then > rests;
    piece = last ? rests : piece - rests;
    const int lane = threadIdx.x & 63;
    const HOPL_GLOBAL int32_t* table = (const HOPL_GLOBAL int32_t*)rows.begin;
    int seen = 0;
    for (int base = 0; base < rows.G; base += 64) {
        const int mine = base + lane;
        int b = 0, e = 0;
        if (mine < rows.G) {
            b = clamp_int(table[mine], 0, rows.rows);
            e = clamp_int(table[mine + 1], b, rows.rows);
        }
        const int own = last ? ((e - b) & (step - 1)) != 0 : (e - b) >> shift;
        int scan = own;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int before = __shfl_up(scan, o);
            if (lane >= o) scan += before;
        }
        const uint64_t behind = __ballot(seen + scan > piece);
        if (behind) {
            const int l = __builtin_ctzll(behind);
            const int gb = __builtin_amdgcn_readlane(b, l), ge = __builtin_amdgcn_readlane(e, l);
            const int first = seen + __builtin_amdgcn_readlane(scan, l) - __builtin_amdgcn_readlane(own, l);
            const int64_t at = last ? ge - ((ge - gb) & (step - 1)) : gb + ((int64_t)(piece - first) << shift);
            if (at < gb || at >= ge) return false;        // only where a broken table made the sums overflow
            *g = base + l;
            *r0 = (int)at;
            *r1 = ge - at < step ? ge : (int)at + step;
            return true;
        }
        seen += __builtin_amdgcn_readlane(scan, 63);
    }
    return false;
}

// The rows of group g.
__device__ __forceinline__ void group_rows(const HopRows& rows, int g, int* b, int* e) {
    if (!rows.begin) {
        *b = 0;
        *e = rows.rows;
        return;
    }
    const HOPL_GLOBAL int32_t* table = (const HOPL_GLOBAL int32_t*)rows.begin;
    *b = __builtin_amdgcn_readfirstlane(clamp_int(table[g], 0, rows.rows));
    *e = __builtin_amdgcn_readfirstlane(clamp_int(table[g + 1], *b, rows.rows));
}

}  // namespace hopl
