// Device code that the attention kernels share: tiles of rows in LDS, the matrix unit's operands, and which rows belong to a workgroup.
//
// All products have 32 x 32 results of which a lane holds a column: 16 of its 32 rows, 8 i + 4 (lane / 32) + e in part i, element e.  Scores are
// computed with the loop's rows (keys, or pairs of queries in the gradient to keys) along the accumulator's rows, so that they are, as they stand, the
// second operand of the product that contracts over those rows: softmax and its gradient never leave the registers.
#pragma once

#include <type_traits>

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
    // The first operand of a product over columns: lane l holds row l % 32, chunk 2 step + l / 32.  Places are a number of the lane's, with a constant's bits flipped,
    // and a constant behind it, so that one register holds the addresses of all reads.
    static __device__ __forceinline__ int along_place() {
        const int lane = threadIdx.x & 63, row = lane & 31;
        return row * kLine + (((lane >> 5) ^ swizzle(row)) << 4);
    }
    static __device__ __forceinline__ frag along(const char* s, int place, int step) { return *(const frag*)(s + (place ^ (step * 32))); }
};

__device__ __forceinline__ f32x16 multiply(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 multiply(f32x4 a, f32x4 b, f32x16 c) {
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
    return c;
}

// An accumulator as the second operand of a product over its rows: two parts of 16 rows.  `across` reads the first operand, 16 of a tile's rows and 32 columns.
// bf16: what is rounded here (the softmax's terms, the scores' gradients; their sums stay in 32 bits) puts results 0.0021 to 0.0025 of their size from 64 bits, where rounding the result alone
// would be 0.0016; a second part with what rounding takes off would be nearly half of all products again (two of attention's four operations, six of the gradients' 14).
// bf16: part u holds rows 16 u + 4 (lane / 32) + e and, from element 4 on, 8 more; the transposing read brings the tile's in the same order (16 lanes hold
// four rows of 16 columns each, lane l of them gets column l).  fp32: an element to a product.
template <typename T>
struct Weights;
template <>
struct Weights<bf16> {
    typedef bf16x8 Part;
    Part part[2];
    static __device__ __forceinline__ Part part_of(const f32x16& p, int u) {
        Part r;
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = (bf16)p[8 * u + e];               // to nearest, ties to even
        return r;
    }
    __device__ __forceinline__ explicit Weights(const f32x16& p) {
        part[0] = part_of(p, 0);
        part[1] = part_of(p, 1);
    }
    template <int D>
    static __device__ __forceinline__ int across_place() {
        typedef Tile<bf16, D> L;
        const int lane = threadIdx.x & 63, row = 4 * (lane >> 5) + (lane >> 2 & 3);
        return row * L::kLine + (((lane >> 4 & 1) * 2 + (lane >> 1 & 1) ^ L::swizzle(row)) << 4) + (lane & 1) * 8;
    }
    template <int D>
    static __device__ __forceinline__ Part across(const char* s, int place, int unit, int u) {
        union { s16x4 half[2]; bf16x8 all; } a;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const char* at = s + (place ^ (unit * 64 + h * 32)) + (16 * u + 8 * h) * Tile<bf16, D>::kLine;
            a.half[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at);
        }
        return a.all;
    }
    static __device__ __forceinline__ f32x16 add(const Part& a, const Part& b, f32x16 c) { return multiply(a, b, c); }
};
template <>
struct Weights<float> {
    typedef f32x8 Part;
    Part part[2];
    static __device__ __forceinline__ Part part_of(const f32x16& p, int u) {
        Part r;
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = p[8 * u + e];
        return r;
    }
    __device__ __forceinline__ explicit Weights(const f32x16& p) {
        part[0] = part_of(p, 0);
        part[1] = part_of(p, 1);
    }
    template <int D>
    static __device__ __forceinline__ int across_place() {
        const int lane = threadIdx.x & 63, hi = lane >> 5;
        return 4 * hi * Tile<float, D>::kLine + (((lane & 31) >> 2 ^ hi << 3) << 4) + (lane & 3) * 4;
    }
    template <int D>
    static __device__ __forceinline__ Part across(const char* s, int place, int unit, int u) {
        Part a;
#pragma unroll
        for (int r = 0; r < 8; ++r) a[r] = *(const float*)(s + (place ^ (unit * 128 + r * 16)) + (16 * u + 8 * (r >> 2) + (r & 3)) * Tile<float, D>::kLine);
        return a;
    }
    static __device__ __forceinline__ f32x16 add(const Part& a, const Part& b, f32x16 c) {
#pragma unroll
        for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
        return c;
    }
};

// Places of operands, worked out again for every unit: held over a loop they would fill the registers.
template <typename T, int D>
struct Places {
    int along = Tile<T, D>::along_place(), across = Weights<T>::template across_place<D>();
    __device__ __forceinline__ Places again() const {
        Places p = *this;
        asm volatile("" : "+v"(p.along), "+v"(p.across));
        return p;
    }
};

template <int N, int I = 0, typename F>
__device__ __forceinline__ void static_for(F f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>());
        static_for<N, I + 1>(f);
    }
}

// ---- products in turn with other things -----------------------------------------------------
// Left to itself the compiler reads an operand right in front of the product that wants it, so that every product waits for LDS, and puts all arithmetic behind
// all products.  Here the order is written down: operands are read kAhead products early, and between two of them the matrix unit has a share of other work beside it.
//
// sum[column][.] += sum over 32 rows of a tile times w.  `begin` reads the first operands.
template <typename T, int D>
struct Sums {
    typedef Weights<T> W;
    static constexpr int kU = D / 32, kN = kU * 2, kAhead = sizeof(T) == 4 ? 2 : kN < 6 ? kN : 6;
    typename W::Part a[kAhead];
    // Products in an order in which neighbours have different sums.
    static __device__ __forceinline__ typename W::Part read(const char* s, int place, int k) { return W::template across<D>(s, place, (k >> 2) * 2 + (k & 1), k >> 1 & 1); }
    __device__ __forceinline__ void begin(const char* s, int place) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k) a[k] = read(s, place, k);
    }
    __device__ __forceinline__ void add(const char* s, int place, const W& w, f32x16* sum) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int k = 0; k < kN; ++k) {
            f32x16& c = sum[(k >> 2) * 2 + (k & 1)];
            c = W::add(a[k % kAhead], w.part[k >> 1 & 1], c);
            if (k + kAhead < kN) a[k % kAhead] = read(s, place, k + kAhead);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
};

// ---- from memory to tiles ---------------------------------------------------------------
// Where the rows of a tile lie: rows of keys, `ld` apart; or pairs, whose group's heads lie beside each other in a row.
struct Rows {
    int64_t ld;
    int group;
    uint32_t inverse;                           // of the group, see hopa_divide
    int shift;
    int cols;
};

// FED: addresses and distances are multiples of 16 bytes, and so are the heads: the memory unit fills the tile itself, through a buffer descriptor whose end
// is that of the rows that there are (what lies outside comes back as zero).  Else, rows of keys only, through registers, by 128-bit loads at an element's address.
// A lane's places in a tile are worked out once, and for pairs again where a tile begins with another head than the one before.
template <typename T, int D, int ROWS, int NT, bool FED, bool PAIRS>
struct Feed {
    typedef Tile<T, D> L;
    static constexpr int kLoads = ROWS * L::kPlaces / NT;
    static_assert(ROWS <= kHopaMostTileRows, "their distance");
    static_assert(FED || !PAIRS, "pairs come from aligned rows");
    uint32_t place[kLoads];                     // FED: bytes behind the tile's first row; else elements
    typename L::frag held[FED ? 1 : kLoads];
    int rest;

    // NT of 64: a wavefront fills a tile of its own
    static __device__ __forceinline__ int thread() { return NT == 64 ? threadIdx.x & 63 : threadIdx.x; }
    static __device__ __forceinline__ int line(int i) { return (i * NT + thread()) / L::kPlaces; }
    static __device__ __forceinline__ int chunk(int i) {
        const int j = i * NT + thread();
        return FED ? (j % L::kPlaces) ^ L::swizzle(j / L::kPlaces) : j % L::kPlaces;
    }
    // rest_: how many heads of the first row belong to pairs in front of the tile
    __device__ __forceinline__ void begin(const Rows& g, int rest_) {
        rest = rest_;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int l = line(i), c = chunk(i) * L::kChunk, row = PAIRS ? hopa_divide(rest + l, g.inverse, g.shift) : l;
            const uint32_t at = (uint32_t)row * (uint32_t)g.ld + (PAIRS ? (rest + l - row * g.group) * g.cols : 0) + c;
            place[i] = FED ? (c >= g.cols ? kOutside : at * (uint32_t)sizeof(T)) : at;
        }
    }
    // rows first, first + 1, ... (numbers of rows, or of pairs), `count` (at least 1) of them exist; base: row 0's first column of the head or the group
    __device__ __forceinline__ void issue(char* stage, const T* base, const Rows& g, int first, int count) {
        const int row0 = PAIRS ? hopa_divide(first, g.inverse, g.shift) : first;
        if (PAIRS && first - row0 * g.group != rest) begin(g, first - row0 * g.group);
        const T* from = base + row0 * g.ld;
        if (count > ROWS) count = ROWS;
        if constexpr (FED) {
            const int64_t end = PAIRS ? hopa_divide(rest + count - 1, g.inverse, g.shift) * g.ld + g.group * g.cols : (count - 1) * g.ld + g.cols;
            const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)from, 0, (int)(end * sizeof(T)), 0x00020000);
            const int wave = thread() >> 6;
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(stage + (i * NT + wave * 64) * 16), 16, place[i], 0, 0, 0);
        } else {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int n = line(i) < count ? g.cols - chunk(i) * L::kChunk : 0;
                held[i] = (T)0.f;
                if (n >= L::kChunk) held[i] = *(const HOPL_GLOBAL typename L::frag_any*)(from + place[i]);
                else if (n > 0) held[i] = load_short<typename L::frag>(from + place[i], n);
            }
        }
    }
    __device__ __forceinline__ void put(char* stage) {
        if constexpr (!FED) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) *(typename L::frag*)(stage + line(i) * L::kLine + ((chunk(i) ^ L::swizzle(line(i))) << 4)) = held[i];
        }
    }
};

// ---- rows that the memory unit cannot take, laid out anew -----------------------------------------
// It fills tiles 16 bytes at a time, from addresses that are multiples of them.  Matrices whose rows or heads are not get a copy with heads of whole 16 bytes (zeros
// at the end): read and written once, in one launch, beside the passes over them that follow.
namespace {
template <typename T>
__global__ __launch_bounds__(256) void attention_align_kernel(HopAttentionCopies c) {
    typedef Tile<T, 64> L;                      // of which only the chunks matter
    const auto& m = c.of[blockIdx.y];
    const int chunks = c.head / L::kChunk, per_row = m.heads * chunks;
    int b = 0, e = m.rows;
    if (m.begin) {
        b = clamp_int(((const HOPL_GLOBAL int32_t*)m.begin)[0], 0, m.rows);
        e = clamp_int(((const HOPL_GLOBAL int32_t*)m.begin)[c.S], b, m.rows);
    }
    const int64_t all = (int64_t)(e - b) * per_row;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int64_t row = b + i / per_row;
        const int at = (int)(i % per_row), head = at / chunks, column = at % chunks * L::kChunk, n = c.cols - column;
        const T* from = (const T*)m.from + row * m.ld + head * c.cols + column;
        typename L::frag v;
        if (n >= L::kChunk) v = *(const HOPL_GLOBAL typename L::frag_any*)from;
        else v = load_short<typename L::frag>(from, n);
        *(HOPL_GLOBAL typename L::frag*)((T*)m.to + row * m.heads * c.head + head * c.head + column) = v;
    }
}
template <typename T>
void launch_copies(const HopAttentionCopies& c, hipStream_t stream) {
    if (!c.n) return;
    int64_t most = 1;
    for (int i = 0; i < c.n; ++i) {
        const int64_t blocks = ((int64_t)c.of[i].rows * c.of[i].heads * c.head * (int64_t)sizeof(T) / 16 + 255) / 256;
        most = most < blocks ? blocks : most;
    }
    attention_align_kernel<T><<<dim3((unsigned)(most < 2048 ? most : 2048), (unsigned)c.n), dim3(256), 0, stream>>>(c);
}
}  // namespace
struct Planner {
    HopAttentionTask& t;
    HopAttentionPlan& p;
    char* scratch;
    int elem;
    Planner(HopAttentionTask* task, HopAttentionPlan* plan, int dtype, char* scratch_) : t(*task), p(*plan), scratch(scratch_), elem(dtype == HOP_BF16 ? 2 : 4) {
        t.head = p.copies.cols = t.cols;
        p.copies.S = t.S;
    }
    char* take(size_t bytes) {
        char* at = (char*)((uintptr_t)scratch + p.bytes);
        p.bytes += (bytes + 255) / 256 * 256;
        return at;
    }
    bool fits(const void* m, int64_t ld) const { return ((uintptr_t)m & 15u) == 0 && (ld * elem) % 16 == 0 && (t.cols * elem) % 16 == 0; }
    // a pointer of the task's and its distance
    template <typename P>
    void align(P& m, int64_t& ld, int rows, int heads, const int32_t* begin) {
        auto& c = p.copies;
        t.head = c.head = (t.cols * elem + 15) / 16 * 16 / elem;
        if (!rows || fits(m, ld)) return;
        char* to = take((size_t)rows * heads * t.head * elem);
        c.of[c.n++] = {m, to, ld, begin, rows, heads};
        m = to;
        ld = (int64_t)heads * t.head;
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

// The same from a tile: a few loads of whole rows are far quicker than a load of every row's chunk by a lane of its own.
template <typename T, int D>
__device__ __forceinline__ void take_columns(typename Tile<T, D>::frag* to, const char* tile, int place) {
#pragma unroll
    for (int s = 0; s < Tile<T, D>::kSteps; ++s) to[s] = Tile<T, D>::along(tile, place, s);
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
    float nothing[4] = {0.f, 0.f, 0.f, 0.f};    // and NaN where it is not
#pragma unroll
    for (int t = 0; t < N; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) nothing[e & 3] = __builtin_fmaf(acc[t][e], 0.f, nothing[e & 3]);
    return (nothing[0] + nothing[1]) + (nothing[2] + nothing[3]) == 0.f;
}
// COLS columns from `column` on, of rows from `from` to `count`; seen(j): whether the lane's column sees row j of the tile
template <typename T, int D, int COLS, typename SEEN>
__device__ __forceinline__ void add_not_finite(const char* s, int column, int from, int count, f32x16 (&acc)[COLS / 32], SEEN seen) {
    typedef Tile<T, D> L;
    const int hi = (threadIdx.x & 63) >> 5;
    for (int j = from; j < count; ++j) {
        const bool here = seen(j);
#pragma unroll
        for (int t = 0; t < COLS / 32; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int c = column + 32 * t + 8 * (e >> 2) + 4 * hi + (e & 3);
                const float v = (float)*(const T*)(s + j * L::kLine + (((c / L::kChunk) ^ L::swizzle(j)) << 4) + c % L::kChunk * sizeof(T));
                acc[t][e] += here && !(__builtin_fabsf(v) < kInf) ? v : 0.f;
            }
    }
}
template <typename T, int BYTES, int NT>
__device__ __forceinline__ void drop_not_finite(char* s) {
    for (int i = NT == 64 ? threadIdx.x & 63 : threadIdx.x; i < BYTES / (int)sizeof(T); i += NT)
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

// Tile number `tile` of the sequences' rows, 1 << shift (times `by` a row) to a tile: its sequence and first row (or pair).  False: there are fewer.
// Every wavefront works it out for itself, 64 sequences at a time, and within those in the order of the place in the sequence, the farthest first: where queries
// see what is in front of them those have most to do, and what begins last is to be short.
__device__ __forceinline__ bool find_tile(const int32_t* begin, int S, int rows, int by, int shift, int tile, int* s, int* first) {
    const int lane = threadIdx.x & 63, step = 1 << shift;
    int seen = 0;
    for (int base = 0; base < S; base += 64) {
        int b = 0, n = 0;
        if (base + lane < S) rows_of(begin, base + lane, rows, &b, &n);
        const int tiles = (int)(((int64_t)n * by + step - 1) >> shift);
        int scan = tiles;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int before = __shfl_up(scan, o);
            if (lane >= o) scan += before;
        }
        const int all = __builtin_amdgcn_readlane(scan, 63);
        if (tile - seen >= all) {
            seen += all;
            continue;
        }
        if (S == 1) {
            const uint64_t behind = __ballot(seen + scan > tile);
            if (!behind) return false;                        // only where a broken table made the sums overflow
            const int l = __builtin_ctzll(behind), its = __builtin_amdgcn_readlane(tiles, l);
            const int at = tile - (seen + __builtin_amdgcn_readlane(scan, l) - its);
            if (at < 0 || at >= its) return false;
            *s = base + l;
            *first = (its - 1 - at) << shift;
            return true;
        }
        // the deepest place from which on there are more tiles than that
        auto from = [&](int depth) {
            int k = tiles > depth ? tiles - depth : 0;
#pragma unroll
            for (int o = 32; o; o >>= 1) k += __shfl_xor(k, o);
            return __builtin_amdgcn_readfirstlane(k);
        };
        const int at = tile - seen;
        int low = 0, high = 1;                                // from(low) > at >= from(high)
        int behind_high;
        while ((behind_high = from(high)) > at) {
            low = high;
            high = high < 1 << 29 ? 2 * high : 0x7FFFFFFF;
        }
        while (high - low > 1) {
            const int middle = low + (high - low) / 2, k = from(middle);
            if (k > at) low = middle;
            else {
                high = middle;
                behind_high = k;
            }
        }
        uint64_t there = __ballot(tiles > low);
        int l = -1;
        for (int skip = at - behind_high; there; there &= there - 1)
            if (skip-- == 0) {
                l = __builtin_ctzll(there);
                break;
            }
        if (l < 0) return false;
        *s = base + l;
        *first = low << shift;
        return true;
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


// ---- stages -----------------------------------------------------------------------------------
// n stages through two buffers, one barrier a stage: the next one is on its way while a stage is worked on.  The buffers are two restricted pointers, so that the
// compiler knows that reads of one need not wait for loads into the other.
template <typename ISSUE, typename WORK>
__device__ __forceinline__ void stage(char* __restrict now, char* __restrict next, int i, int n, ISSUE issue, WORK work) {
    if (i + 1 < n) issue(next, i + 1);
    work(now, i);
}
// The first one is issued beforehand, behind a barrier with whoever still reads from the buffers.
template <typename ISSUE, typename WORK>
__device__ __forceinline__ void stages(int n, char* pool, int bytes, ISSUE issue, WORK work) {
    char *now = pool, *next = pool + bytes;
    for (int i = 0; i < n; ++i) {
        arrive();                               // this stage is there, and nobody reads from the one before any more
        stage(now, next, i, n, issue, work);
        char* const other = now;
        now = next;
        next = other;
    }
}

// ---- even shares ------------------------------------------------------------------------------
// Tiles of sequences of any lengths, weighed in stages and what a tile takes beside them, laid end to end and cut into as many equal runs as there are workgroups: a run
// is the end of a tile, whole tiles and the beginning of another.  What does not cover its tile is left as a part, and the parts of a tile are added in their order.
struct PlanTile {
    int64_t before;                             // weight in front of it
    int32_t q0, nq, k0, nk, first, stages;
};
struct Plan {
    int64_t weight;                             // of a head's tiles
    int64_t tiles;
    int64_t fixed;                              // stages that a tile's operands and its sums' way out are worth
    PlanTile tile[1];                           // tiles + 1 of them
};
constexpr int kLeast = 4;                       // stages: a run has that many, and no cut lies nearer to the edge of a tile

struct Runs {
    const HOPL_GLOBAL Plan* plan;
    int64_t all;                                // weight of all heads
    int64_t blocks;
    int fixed;
    __device__ __forceinline__ Runs(const void* p, int heads, int most) : plan((const HOPL_GLOBAL Plan*)p) {
        fixed = (int)plan->fixed;
        all = plan->weight * heads;
        blocks = all / kLeast;
        blocks = blocks < 1 ? 1 : blocks > most ? most : blocks;
    }
};
__device__ __forceinline__ PlanTile tile_of(const Runs& r, int64_t number) {
    const HOPL_GLOBAL PlanTile* t = &r.plan->tile[number];
    auto same = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    return {t->before, same(t->q0), same(t->nq), same(t->k0), same(t->nk), same(t->first), same(t->stages)};
}
struct Place {
    int64_t tile;                               // head * tiles + number
    int stage;
};
// Where the run of workgroup `block` begins: the same for all wavefronts, which search 64 tiles at a time.
__device__ __forceinline__ Place begin_of_run(const Runs& r, int64_t block) {
    const int64_t tiles = r.plan->tiles;
    const int64_t w = block * r.all / r.blocks;
    if (!r.all || w >= r.all) return {r.all / (r.plan->weight ? r.plan->weight : 1) * tiles, 0};
    const int64_t head = w / r.plan->weight, in = w - head * r.plan->weight;
    int64_t low = 0, high = tiles;              // tile[low].before <= in < tile[high].before
    while (high - low > 1) {
        const int64_t step = (high - low + 63) / 64, at = low + (threadIdx.x & 63) * step;
        const uint64_t before = __ballot(at < high && r.plan->tile[at].before <= in);
        low += (63 - __builtin_clzll(before)) * step;
        high = low + step < high ? low + step : high;
    }
    const int stage = (int)(in - r.plan->tile[low].before) - r.fixed, stages = r.plan->tile[low].stages;
    if (stage < kLeast) return {head * tiles + low, 0};
    if (stages - stage < kLeast) return {head * tiles + low + 1, 0};
    return {head * tiles + low, stage};
}
// The workgroups whose runs begin inside of a tile, from *first to *last; false: none does.
__device__ __forceinline__ bool runs_inside(const Runs& r, int64_t head, const PlanTile& tile, int64_t* first, int64_t* last) {
    if (tile.stages < 2 * kLeast) return false;
    const int64_t at = head * r.plan->weight + tile.before + r.fixed, from = at + kLeast, to = at + tile.stages - kLeast + 1;    // [from, to)
    *first = (from * r.blocks + r.all - 1) / r.all;
    *last = (to * r.blocks + r.all - 1) / r.all - 1;
    return *first <= *last;
}

}  // namespace hopa
