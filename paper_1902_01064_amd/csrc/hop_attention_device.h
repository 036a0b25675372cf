// Device code that the attention kernels share: tiles of rows in LDS, the matrix unit's operands, and which rows belong to a workgroup.
//
// All products have 32 x 32 results of which a lane holds a column: 16 of its 32 rows, 8 i + 4 (lane / 32) + e in part i, element e.  Scores are
// computed with the loop's rows (keys, or pairs of queries in the gradient to keys) along the accumulator's rows, so that they are, as they stand, the
// second operand of the product that contracts over those rows: softmax and its gradient never leave the registers.
#pragma once

#include "hop_attention_internal.h"
#include "hop_layers_device.h"

namespace hopa {

using namespace hopl;

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float kInf = __builtin_huge_valf();
constexpr float kLn2 = 0.693147180559945309f;
constexpr uint32_t kOutside = 0x80000000u;      // beyond any descriptor's end

// ---- tiles in LDS -----------------------------------------------------------------------
// Rows of D columns in 16-byte chunks; chunk c of row r stands at place c ^ swizzle(r), so that neither 16 rows read at one chunk nor
// (transposed) 4 or 8 rows read at 64 consecutive bytes meet in a bank.
template <typename T, int D>
struct Tile {
    static constexpr int kLine = D * (int)sizeof(T), kPlaces = kLine / 16, kChunk = 16 / (int)sizeof(T), kSteps = kPlaces / 2;
    static constexpr int kUnits = D / 32;                  // of 32 columns
    typedef T frag __attribute__((ext_vector_type(kChunk)));
    typedef frag frag_any __attribute__((aligned(sizeof(T))));

    static __device__ __forceinline__ int swizzle(int r) {
        if (sizeof(T) == 4) return ((r >> 2 & 1) << 3) | (r & 3) | (r >> 1 & 4);
        if (kLine == 128) return ((r >> 1 & 1) << 2) | (r >> 2 & 3);
        return ((r & 3) << 2) | (r >> 2 & 3);
    }
    // The first operand of a product over columns: lane l holds row l % 32, chunk 2 step + l / 32.
    static __device__ __forceinline__ frag along(const char* s, int row0, int step) {
        const int lane = threadIdx.x & 63, row = row0 + (lane & 31), c = step * 2 + (lane >> 5);
        return *(const frag*)(s + row * kLine + ((c ^ swizzle(row)) << 4));
    }
};

__device__ __forceinline__ f32x16 multiply(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 multiply(f32x4 a, f32x4 b, f32x16 c) {
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
    return c;
}

// An accumulator as the second operand of a product over its rows, and that product: c[column][.] += sum over 32 rows of a tile from row0 on.
// bf16: part u holds rows 16 u + 4 (lane / 32) + e and, from element 4 on, 8 more; the transposing read brings the tile's in the same order (16 lanes hold
// four rows of 16 columns each, lane l of them gets column l).
template <typename T>
struct Weights;
template <>
struct Weights<bf16> {
    bf16x8 part[2];
    __device__ __forceinline__ explicit Weights(const f32x16& p) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) part[u][e] = (bf16)p[8 * u + e];     // to nearest, ties to even
    }
    template <int D>
    __device__ __forceinline__ f32x16 product(const char* s, int row0, int unit, f32x16 c) const {
        typedef Tile<bf16, D> L;
        const int lane = threadIdx.x & 63, col = 32 * unit + (lane & 16) + (lane & 3) * 4;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            union { s16x4 half[2]; bf16x8 all; } a;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = row0 + 16 * u + 8 * h + 4 * (lane >> 5) + (lane >> 2 & 3);
                const char* at = s + row * L::kLine + (((col >> 3) ^ L::swizzle(row)) << 4) + (col & 4) * 2;
                a.half[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at);
            }
            c = multiply(a.all, part[u], c);
        }
        return c;
    }
};
template <>
struct Weights<float> {
    f32x16 p;
    __device__ __forceinline__ explicit Weights(const f32x16& p_) : p(p_) {}
    template <int D>
    __device__ __forceinline__ f32x16 product(const char* s, int row0, int unit, f32x16 c) const {
        typedef Tile<float, D> L;
        const int lane = threadIdx.x & 63, col = 32 * unit + (lane & 31);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int row = row0 + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3);
            const float a = *(const float*)(s + row * L::kLine + (((col >> 2) ^ L::swizzle(row)) << 4) + (col & 3) * 4);
            c = __builtin_amdgcn_mfma_f32_32x32x2f32(a, p[r], c, 0, 0, 0);
        }
        return c;
    }
};

// ---- from memory to tiles ---------------------------------------------------------------
__device__ __forceinline__ int divide(int x, uint32_t inverse) { return inverse ? (int)__umulhi((uint32_t)x, inverse) : x; }

// Where the rows of a tile lie: rows of keys, `ld` apart; or pairs, whose group's heads lie beside each other in a row.
struct Rows {
    int64_t ld;
    int group;
    uint32_t inverse;
    int cols;
};

// FED: addresses and distances are multiples of 16 bytes, and so are the heads: the memory unit fills the tile itself, through a buffer descriptor whose end
// is that of the rows that there are (what lies outside comes back as zero).  Else through registers, by 128-bit loads at an element's address.
template <typename T, int D, int ROWS, int NT, bool FED, bool PAIRS>
struct Feed {
    typedef Tile<T, D> L;
    static constexpr int kLoads = ROWS * L::kPlaces / NT;
    typename L::frag held[FED ? 1 : kLoads];

    // rows first, first + 1, ... (numbers of rows, or of pairs), `count` (at least 1) of them exist; base: row 0's first column of the head or the group
    __device__ __forceinline__ void issue(char* stage, const T* base, const Rows& g, int first, int count) {
        const int row0 = PAIRS ? divide(first, g.inverse) : first, rest = PAIRS ? first - row0 * g.group : 0;
        const T* from = base + row0 * g.ld;
        if (count > ROWS) count = ROWS;
        if constexpr (FED) {
            const int64_t end = PAIRS ? divide(rest + count - 1, g.inverse) * g.ld + g.group * g.cols : (count - 1) * g.ld + g.cols;
            const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)from, 0, (int)(end * sizeof(T)), 0x00020000);
            const int wave = threadIdx.x >> 6;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int j = i * NT + threadIdx.x, l = j / L::kPlaces, c = (j % L::kPlaces) ^ L::swizzle(l);
                const int row = PAIRS ? divide(rest + l, g.inverse) : l;
                uint32_t o = (uint32_t)(row * (uint32_t)g.ld + (PAIRS ? (rest + l - row * g.group) * g.cols : 0)) * sizeof(T) + c * 16;
                if (c * L::kChunk >= g.cols || l >= count) o = kOutside;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(stage + (i * NT + wave * 64) * 16), 16, o, 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int j = i * NT + threadIdx.x, l = j / L::kPlaces, c = j % L::kPlaces * L::kChunk, n = g.cols - c;
                const int row = PAIRS ? divide(rest + l, g.inverse) : l;
                held[i] = (T)0.f;
                if (l >= count || n <= 0) continue;
                const T* p = from + row * g.ld + (PAIRS ? (rest + l - row * g.group) * g.cols : 0) + c;
                if (n >= L::kChunk) held[i] = *(const HOPL_GLOBAL typename L::frag_any*)p;
                else held[i] = load_short<typename L::frag>(p, n);
            }
        }
    }
    __device__ __forceinline__ void put(char* stage) {
        if constexpr (!FED) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int j = i * NT + threadIdx.x, l = j / L::kPlaces, c = (j % L::kPlaces) ^ L::swizzle(l);
                *(typename L::frag*)(stage + l * L::kLine + c * 16) = held[i];
            }
        }
    }
};

// A lane's column of the second operand: its row's chunks 2 step + lane / 32, zeros where there is no row.
template <typename T, int D, bool FED>
__device__ __forceinline__ void load_columns(typename Tile<T, D>::frag* to, const T* row, int cols, bool live) {
    typedef Tile<T, D> L;
#pragma unroll
    for (int s = 0; s < L::kSteps; ++s) {
        const int c = (2 * s + (int)((threadIdx.x & 63) >> 5)) * L::kChunk, n = live ? cols - c : 0;
        to[s] = (T)0.f;
        if (n >= L::kChunk) {
            if constexpr (FED) to[s] = *(const HOPL_GLOBAL typename L::frag*)(row + c);
            else to[s] = *(const HOPL_GLOBAL typename L::frag_any*)(row + c);
        } else if (!FED && n > 0) {
            to[s] = load_short<typename L::frag>(row + c, n);
        }
    }
}

__device__ __forceinline__ void store4(float* p, int n, f32x4 v) {
    if (n >= 4) {
        *(HOPL_GLOBAL f32x4_any*)p = v;
        return;
    }
#pragma unroll
    for (int i = 0; i < 3; ++i)
        if (i < n) ((HOPL_GLOBAL float*)p)[i] = v[i];
}
__device__ __forceinline__ void store4(bf16* p, int n, f32x4 v) {
    const bf16x4 r = __builtin_convertvector(v, bf16x4);      // to nearest, ties to even
    if (n >= 4) {
        *(HOPL_GLOBAL bf16x4_any*)p = r;
        return;
    }
#pragma unroll
    for (int i = 0; i < 3; ++i)
        if (i < n) ((HOPL_GLOBAL bf16*)p)[i] = r[i];
}
// A lane's column of an accumulator of D rows, times `by`, to its row of the result.
template <typename OUT, int D>
__device__ __forceinline__ void store_columns(OUT* row, int cols, const f32x16 (&acc)[D / 32], float by) {
    const int hi = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = 32 * t + 8 * i + 4 * hi;
            f32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = acc[t][4 * i + e] * by;
            if (at < cols) store4(row + at, cols - at, v);
        }
}

// Everything before has arrived, in this wavefront and in the workgroup's others.
__device__ __forceinline__ void arrive() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070);         // vmcnt(0) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// The value of the lane that holds the other half of this lane's column, combined.
__device__ __forceinline__ float both_max(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float both_sum(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// ---- what a column does not see -----------------------------------------------------------
// Rows of a tile that a column does not see have weight zero, which infinities and NaN in them would turn into NaN.  They are looked for only where
// a result is not finite: then the workgroup starts again, and in tiles that some column sees in part it adds what is not finite by hand, where it is seen,
// and sets it to zero in the tile before the matrix unit reads it.
template <int N>
__device__ __forceinline__ bool all_finite(const f32x16 (&acc)[N]) {
    bool fine = true;
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) fine = fine && __builtin_fabsf(acc[t][e]) < kInf;
    return fine;
}
// seen(j): whether the lane's column sees row j of the tile
template <typename T, int D, typename SEEN>
__device__ __forceinline__ void add_not_finite(const char* s, int count, f32x16 (&acc)[D / 32], SEEN seen) {
    typedef Tile<T, D> L;
    const int hi = (threadIdx.x & 63) >> 5;
    for (int j = 0; j < count; ++j) {
        const bool here = seen(j);
#pragma unroll
        for (int t = 0; t < D / 32; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int c = 32 * t + 8 * (e >> 2) + 4 * hi + (e & 3);
                const float v = (float)*(const T*)(s + j * L::kLine + (((c / L::kChunk) ^ L::swizzle(j)) << 4) + c % L::kChunk * sizeof(T));
                acc[t][e] += here && !(__builtin_fabsf(v) < kInf) ? v : 0.f;
            }
    }
}
template <typename T, int BYTES, int NT>
__device__ __forceinline__ void drop_not_finite(char* s) {
    for (int i = threadIdx.x; i < BYTES / (int)sizeof(T); i += NT)
        if (!(__builtin_fabsf((float)((T*)s)[i]) < kInf)) ((T*)s)[i] = (T)0.f;
}

// ---- which rows -----------------------------------------------------------------------------
struct Sequence {
    int q0, nq, k0, nk;
};
__device__ __forceinline__ void rows_of(const int32_t* begin, int s, int rows, int* b, int* n) {
    if (!begin) {
        *b = 0;
        *n = rows;
        return;
    }
    const HOPL_GLOBAL int32_t* table = (const HOPL_GLOBAL int32_t*)begin;
    *b = clamp_int(table[s], 0, rows);
    *n = clamp_int(table[s + 1], *b, rows) - *b;
}

// Tile number `tile` of the sequences' rows, 1 << shift (times `by` a row) to a tile: its sequence and first row (or pair).  `back`: from the last
// sequence's last tile on.  False: there are fewer.  Every wavefront works it out for itself, 64 sequences at a time.
__device__ __forceinline__ bool find_tile(const int32_t* begin, int S, int rows, int by, int shift, bool back, int tile, int* s, int* first) {
    const int lane = threadIdx.x & 63, step = 1 << shift;
    int seen = 0;
    for (int base = 0; base < S; base += 64) {
        const int mine = back ? S - 1 - (base + lane) : base + lane;
        int b = 0, n = 0;
        if (base + lane < S) rows_of(begin, mine, rows, &b, &n);
        const int tiles = (int)(((int64_t)n * by + step - 1) >> shift);
        int scan = tiles;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int before = __shfl_up(scan, o);
            if (lane >= o) scan += before;
        }
        const uint64_t behind = __ballot(seen + scan > tile);
        if (behind) {
            const int l = __builtin_ctzll(behind), its = __builtin_amdgcn_readlane(tiles, l);
            const int at = tile - (seen + __builtin_amdgcn_readlane(scan, l) - its);
            if (at < 0 || at >= its) return false;            // only where a broken table made the sums overflow
            *s = back ? S - 1 - (base + l) : base + l;
            *first = (back ? its - 1 - at : at) << shift;
            return true;
        }
        seen += __builtin_amdgcn_readlane(scan, 63);
    }
    return false;
}

__device__ __forceinline__ Sequence sequence(const HopAttentionTask& t, int s) {
    Sequence q;
    rows_of(t.q_begin, s, t.q_rows, &q.q0, &q.nq);
    rows_of(t.k_begin, s, t.k_rows, &q.k0, &q.nk);
    q.q0 = __builtin_amdgcn_readfirstlane(q.q0);
    q.nq = __builtin_amdgcn_readfirstlane(q.nq);
    q.k0 = __builtin_amdgcn_readfirstlane(q.k0);
    q.nk = __builtin_amdgcn_readfirstlane(q.nk);
    return q;
}
// How many keys of its sequence a row of queries sees.
__device__ __forceinline__ int visible(const Sequence& q, int causal, int row) { return causal ? clamp_int(row + 1 + q.nk - q.nq, 0, q.nk) : q.nk; }

}  // namespace hopa
