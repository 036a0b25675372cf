// Products of rows grouped by worker or expert with their group's weights, and the gradient to the weights, for gfx950.
#include "hop_layers_device.h"

using namespace hopl;

namespace {

#ifndef HOPL_BM
#define HOPL_BM 256
#define HOPL_BN 256
#define HOPL_WM 2
#define HOPL_WN 4
#endif
constexpr int kTile = 64;               // rows and columns of a workgroup's tile
constexpr int kStep = 32;               // of the contraction per turn
constexpr int kThreads = 256;

typedef short s16x4 __attribute__((ext_vector_type(4)));

template <typename T>
struct Raw;                             // eight elements as they are
template <>
struct Raw<bf16> { typedef bf16x8 type; typedef bf16x8_any any; };
template <>
struct Raw<float> { typedef f32x8 type; typedef f32x8_any any; };

template <typename T>
__device__ __forceinline__ typename Raw<T>::type raw8(const T* p, int n) {
    if (n >= 8) return *(const HOPL_GLOBAL typename Raw<T>::any*)p;
    typename Raw<T>::type v = (T)0.f;
#pragma unroll
    for (int i = 0; i < 7; ++i)
        if (i < n) v[i] = ((const HOPL_GLOBAL T*)p)[i];
    return v;
}

// One operand of a tile, kTile lines (rows or columns of the result) by kStep of the contraction.  ALONG: the contraction is
// contiguous in memory (element (line, k) at p[line * ld + k]), else the lines are (p[k * ld + line]); it lies in LDS as in memory.
// What lies outside the operand is zero in LDS: a neighbouring group's rows never meet this group's sums, whatever they hold.
template <typename T, bool ALONG>
struct Operand {
    static constexpr int kPad = 16 / sizeof(T);
    static constexpr int kLd = (ALONG ? kStep : kTile) + kPad;
    static constexpr int kElems = (ALONG ? kTile : kStep) * kLd;
    typename Raw<T>::type part;

    __device__ __forceinline__ void load(const T* p, int64_t ld, int lines, int k0, int K) {
        const int a = ALONG ? threadIdx.x >> 2 : threadIdx.x >> 3;
        const int b = ALONG ? (threadIdx.x & 3) * 8 : (threadIdx.x & 7) * 8;
        const int have_a = ALONG ? lines : K - k0, have_b = ALONG ? K - k0 : lines;
        part = (T)0.f;
        if (a < have_a && b < have_b)
            part = raw8(ALONG ? p + a * ld + (k0 + b) : p + (int64_t)(k0 + a) * ld + b, have_b - b);
    }
    __device__ __forceinline__ void put(T* s) const {
        const int a = ALONG ? threadIdx.x >> 2 : threadIdx.x >> 3;
        const int b = ALONG ? (threadIdx.x & 3) * 8 : (threadIdx.x & 7) * 8;
        *(typename Raw<T>::type*)(s + a * kLd + b) = part;
    }
};

// acc[i][j]: rows p0 + 16 j + lane % 16, columns q0 + 16 i + 4 (lane / 16) ..: the columns' operand is the first of the matrix
// instruction, so that a lane holds four consecutive columns of one row.
template <bool PA, bool QA>
__device__ __forceinline__ void multiply(const bf16* sp, const bf16* sq, int p0, int q0, f32x4 (&acc)[2][2]) {
    const int lane = threadIdx.x & 63, l16 = lane & 15, quad = lane >> 4;
    bf16x8 p[2], q[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            const bool along = which ? QA : PA;
            const bf16* s = which ? sq : sp;
            const int at = (which ? q0 : p0) + 16 * i;
            bf16x8 v;
            if (along) {
                v = *(const bf16x8*)(s + (at + l16) * Operand<bf16, true>::kLd + quad * 8);
            } else {
                // the transposing read: 16 lanes hold four lines of 16 elements, lane l gets column l of them
                const bf16* a = s + (quad * 8 + (l16 >> 2)) * Operand<bf16, false>::kLd + at + (l16 & 3) * 4;
                union { s16x4 half[2]; bf16x8 all; } u;
                u.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)a);
                u.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(a + 4 * Operand<bf16, false>::kLd));
                v = u.all;
            }
            (which ? q : p)[i] = v;
        }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[i], p[j], acc[i][j], 0, 0, 0);
}

// fp32: 16 x 16 x 4 instructions; the contraction's order is the operands' own affair, so a lane takes four consecutive k.
template <bool PA, bool QA>
__device__ __forceinline__ void multiply(const float* sp, const float* sq, int p0, int q0, f32x4 (&acc)[2][2]) {
    const int lane = threadIdx.x & 63, l16 = lane & 15, quad = lane >> 4;
#pragma unroll
    for (int k = 0; k < kStep; k += 16) {
        f32x4 p[2], q[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int which = 0; which < 2; ++which) {
                const bool along = which ? QA : PA;
                const float* s = which ? sq : sp;
                const int at = (which ? q0 : p0) + 16 * i + l16, k4 = k + quad * 4;
                f32x4 v;
                if (along) {
                    v = *(const f32x4*)(s + at * Operand<float, true>::kLd + k4);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = s[(k4 + e) * Operand<float, false>::kLd + at];
                }
                (which ? q : p)[i] = v;
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(q[i][e], p[j][e], acc[i][j], 0, 0, 0);
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
    const bf16x4 r = __builtin_convertvector(v, bf16x4);
    if (n >= 4) {
        *(HOPL_GLOBAL bf16x4_any*)p = r;
        return;
    }
#pragma unroll
    for (int i = 0; i < 3; ++i)
        if (i < n) ((HOPL_GLOBAL bf16*)p)[i] = r[i];
}

// c[p][q] = sum over k of P(p, k) Q(q, k), one tile of it: `np` rows and `nq` columns exist from here on.
template <typename T, typename OUT, bool PA, bool QA>
__device__ __forceinline__ void tile_product(const T* p, int64_t ldp, int np, const T* q, int64_t ldq, int nq, int K, OUT* c, int64_t ldc) {
    typedef Operand<T, PA> P;
    typedef Operand<T, QA> Q;
    __shared__ __attribute__((aligned(16))) T sp[P::kElems], sq[Q::kElems];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int p0 = (wave & 1) * 32, q0 = (wave >> 1) * 32;
    f32x4 acc[2][2] = {};
    P rp;
    Q rq;
    if (K > 0) {
        rp.load(p, ldp, np, 0, K);
        rq.load(q, ldq, nq, 0, K);
    }
    for (int k = 0; k < K; k += kStep) {
        __syncthreads();
        rp.put(sp);
        rq.put(sq);
        __syncthreads();
        if (K - k > kStep) {
            rp.load(p, ldp, np, k + kStep, K);
            rq.load(q, ldq, nq, k + kStep, K);
        }
        multiply<PA, QA>(sp, sq, p0, q0, acc);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int row = p0 + 16 * j + (lane & 15), col = q0 + 16 * i + 4 * (lane >> 4);
            if (row < np && col < nq) store4(c + row * ldc + col, nq - col, acc[i][j]);
        }
}

// ---- staged tiles -------------------------------------------------------------------
// Tiles of 128 bytes of the contraction, fed to LDS by the memory unit itself (128-bit loads that pass no register) into one of two
// stages while the matrix instructions run on the other.  An operand whose contraction is contiguous (ALONG) lies in LDS line by
// line, eight 16-byte chunks each; one whose lines are contiguous lies there row of the contraction by row.  The memory unit fills
// LDS in the order of the lanes, so what moves to keep the reads off each other's banks is which chunk a lane asks for: chunk c of
// line l stands at place c ^ (l / 2 mod 8); chunk c of row k at c ^ 4 (k mod 4) in 16 bits, c ^ 4 (k / 4 mod 4) in 32.  The loads go through a buffer descriptor whose end is the operand's: what lies outside comes back as zero.
constexpr int kStepBytes = 128;
constexpr uint32_t kOutside = 0x80000000u;      // beyond any descriptor's end

template <typename T, bool ALONG, int LINES, int NT>
struct Feed {
    static constexpr int kChunk = 16 / sizeof(T);                       // elements
    static constexpr int kK = kStepBytes / sizeof(T);                   // of the contraction per stage
    static constexpr int kPerLine = ALONG ? 8 : LINES / kChunk;         // chunks of a line (or row of the contraction) in LDS
    static constexpr int kLoads = LINES * 8 / NT;
    static constexpr int kBytes = LINES * kStepBytes;
    const char* base;
    int64_t ld;
    int lines, K;
    uint32_t off[kLoads];
    int first[ALONG ? kLoads : 1];              // place in the contraction of each load's chunk, ALONG only

    static __device__ __forceinline__ int swizzle(int l) {
        if (ALONG) return (l >> 1) & 7;
        return sizeof(T) == 2 ? (l & 3) << 2 : ((l >> 2) & 3) << 2;
    }
    __device__ __forceinline__ void start(const T* p, int64_t ld_, int lines_, int K_) {
        base = (const char*)p;
        ld = ld_;
        lines = lines_ < LINES ? lines_ : LINES;
        K = K_;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int j = i * NT + threadIdx.x, l = j / kPerLine, c = (j % kPerLine) ^ swizzle(l);
            off[i] = (uint32_t)(l * ld * sizeof(T)) + c * 16;
            if (ALONG) first[i] = c * kChunk;
            else if (c * kChunk >= lines) off[i] = kOutside;
        }
    }
    __device__ __forceinline__ void issue(char* stage, int k) const {
        const int64_t left = K - k;
        const int64_t end = ALONG ? (lines - 1) * ld + left : ((left < kK ? left : kK) - 1) * ld + lines;
        const __amdgpu_buffer_rsrc_t r =
            __builtin_amdgcn_make_buffer_rsrc((void*)(base + (ALONG ? k : k * ld) * sizeof(T)), 0, (int)(end * sizeof(T)), 0x00020000);
        const int wave = threadIdx.x >> 6;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            uint32_t o = off[i];
            if (ALONG && first[i] >= left) o = kOutside;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(stage + (i * NT + wave * 64) * 16), 16, o, 0, 0, 0);
        }
    }
};

// What a turn of the matrix unit takes.  16 bits: 32 lines by 16 of the contraction (fewer addresses to hold than 16 x 32, which left the
// kernel short of registers); lane l holds line l % 32 and eight of the contraction from 8 (l / 32) on.  32 bits: 16 lines by 16, in four
// instructions; lane l holds line l % 16 and four of the contraction from 4 (l / 16) on.
template <typename T>
struct Unit;
template <>
struct Unit<bf16> {
    static constexpr int kLines = 32, kTurns = 4;
    typedef bf16x8 frag;
    typedef float acc __attribute__((ext_vector_type(16)));
    static __device__ __forceinline__ acc step(frag q, frag p, acc c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(q, p, c, 0, 0, 0); }
    static __device__ __forceinline__ frag along(const char* s, int line0, int turn) {
        const int lane = threadIdx.x & 63, line = line0 + (lane & 31), c = turn * 2 + (lane >> 5);
        return *(const frag*)(s + line * 128 + ((c ^ ((line >> 1) & 7)) << 4));
    }
    template <int LINES>
    static __device__ __forceinline__ frag across(const char* s, int line0, int turn) {
        // the transposing read: 16 lanes hold four rows of the contraction of 16 lines each, lane l of them gets column l
        const int lane = threadIdx.x & 63, line = line0 + (lane & 16) + (lane & 3) * 4, row = (lane & 15) >> 2;
        const int k = turn * 16 + (lane >> 5) * 8 + row, place = (((line >> 3) ^ (row << 2)) << 4) + (line & 4) * 2;
        union { s16x4 half[2]; frag all; } u;
        u.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(s + k * LINES * 2 + place));
        u.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(s + (k + 4) * LINES * 2 + place));
        return u.all;
    }
    // the four columns of part i of an accumulator begin here; its row is the lane's line
    static __device__ __forceinline__ int column(int i) { return 8 * i + 4 * ((threadIdx.x & 63) >> 5); }
};
template <>
struct Unit<float> {
    static constexpr int kLines = 16, kTurns = 2;
    typedef f32x4 frag;
    typedef f32x4 acc;
    static __device__ __forceinline__ acc step(frag q, frag p, acc c) {
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(q[e], p[e], c, 0, 0, 0);
        return c;
    }
    static __device__ __forceinline__ frag along(const char* s, int line0, int turn) {
        const int lane = threadIdx.x & 63, line = line0 + (lane & 15), c = turn * 4 + (lane >> 4);
        return *(const frag*)(s + line * 128 + ((c ^ ((line >> 1) & 7)) << 4));
    }
    template <int LINES>
    static __device__ __forceinline__ frag across(const char* s, int line0, int turn) {
        const int lane = threadIdx.x & 63, line = line0 + (lane & 15), quad = lane >> 4;
        const char* at = s + (turn * 16 + quad * 4) * LINES * 4 + ((((line >> 2) ^ (quad << 2)) << 4) + (line & 3) * 4);
        frag v;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = *(const float*)(at + e * LINES * 4);
        return v;
    }
    static __device__ __forceinline__ int column(int) { return 4 * ((threadIdx.x & 63) >> 4); }
};

// Everything before has arrived, in this wavefront and in the workgroup's others.
__device__ __forceinline__ void arrive() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070);         // vmcnt(0) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

template <typename T, typename OUT, bool PA, bool QA, int BM, int BN, int WM, int WN>
__device__ __forceinline__ void staged_product(const T* p, int64_t ldp, int np, const T* q, int64_t ldq, int nq, int K, OUT* c, int64_t ldc) {
    typedef Unit<T> U;
    constexpr int NT = WM * WN * 64, TM = BM / WM, TN = BN / WN, FM = TM / U::kLines, FN = TN / U::kLines;
    constexpr int kK = kStepBytes / sizeof(T);
    typedef Feed<T, PA, BM, NT> P;
    typedef Feed<T, QA, BN, NT> Q;
    // arrays of their own, so that the compiler knows that reads of one stage need not wait for loads into the other
    __shared__ __attribute__((aligned(16))) char sp0[P::kBytes], sq0[Q::kBytes], sp1[P::kBytes], sq1[Q::kBytes];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int p0 = (wave % WM) * TM, q0 = (wave / WM) * TN;
    typename U::acc acc[FN][FM] = {};
    P fp;
    Q fq;
    fp.start(p, ldp, np, K);
    fq.start(q, ldq, nq, K);
    auto turn = [&](const char* sp, const char* sq) {
#pragma unroll
        for (int t = 0; t < U::kTurns; ++t) {
            typename U::frag a[FM], b[FN];
#pragma unroll
            for (int i = 0; i < FN; ++i) {
                if constexpr (QA) b[i] = U::along(sq, q0 + U::kLines * i, t);
                else b[i] = U::template across<BN>(sq, q0 + U::kLines * i, t);
            }
#pragma unroll
            for (int j = 0; j < FM; ++j) {
                if constexpr (PA) a[j] = U::along(sp, p0 + U::kLines * j, t);
                else a[j] = U::template across<BM>(sp, p0 + U::kLines * j, t);
            }
#pragma unroll
            for (int j = 0; j < FM; ++j)
#pragma unroll
                for (int i = 0; i < FN; ++i) acc[i][j] = U::step(b[i], a[j], acc[i][j]);
            if (t & 1) __builtin_amdgcn_sched_barrier(0);      // fragments of two turns at a time: all at once do not fit the registers
        }
    };
    auto issue = [&](char* sp, char* sq, int step) {
        fp.issue(sp, step * kK);
        fq.issue(sq, step * kK);
    };
    const int steps = (K + kK - 1) / kK;
    if (steps) issue(sp0, sq0, 0);
    int step = 0;
    for (; step + 1 < steps; step += 2) {
        arrive();
        issue(sp1, sq1, step + 1);
        turn(sp0, sq0);
        arrive();
        if (step + 2 < steps) issue(sp0, sq0, step + 2);
        turn(sp1, sq1);
    }
    if (step < steps) {
        arrive();
        turn(sp0, sq0);
    }
#pragma unroll
    for (int j = 0; j < FM; ++j) {
        const int row = p0 + U::kLines * j + (lane & (U::kLines - 1));
        if (row >= np) continue;
        OUT* to = c + row * ldc;
#pragma unroll
        for (int i = 0; i < FN; ++i)
#pragma unroll
            for (int v = 0; v < (int)(sizeof(typename U::acc) / 16); ++v) {
                const int col = q0 + U::kLines * i + U::column(v);
                if (col < nq) store4(to + col, nq - col, f32x4{acc[i][j][4 * v], acc[i][j][4 * v + 1], acc[i][j][4 * v + 2], acc[i][j][4 * v + 3]});
            }
    }
}

// Which tile a workgroup takes: those of one XCD (workgroups are dealt to the 8 of them in turn) lie together, and within them kBand
// pieces of rows are worked through column of tiles by column, so that the operands' tiles are found in that XCD's L2 again.
constexpr int kBand = 4;
__device__ __forceinline__ bool place_tile(int b, int pieces, int columns, int* piece, int* column) {
    const int total = pieces * columns;
    if (b >= total) return false;
    const int each = total / 8, more = total % 8, x = b % 8;
    const int at = x * each + (x < more ? x : more) + b / 8;
    const int band = at / (kBand * columns), within = at - band * kBand * columns;
    const int height = pieces - band * kBand < kBand ? pieces - band * kBand : kBand;
    *column = within / height;
    *piece = band * kBand + within % height;
    return true;
}

template <typename T, bool TRANSPOSED, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM* WN * 64) void product_staged_kernel(HopProductTask t, int columns, HopIndex index) {
    constexpr int shift = BM == 256 ? 8 : BM == 128 ? 7 : 6;
    int piece, column, g, r0, r1;
    if (!place_tile(blockIdx.x, count_pieces(t.rows, shift), columns, &piece, &column)) return;
    if (!find_piece(t.rows, shift, piece, &g, &r0, &r1)) return;
    const int64_t n0 = (int64_t)column * BN;
    const int at = t.indexed ? index.at[g] : g;
    const T* w = (const T*)t.w + at * t.w_stride + (TRANSPOSED ? n0 : n0 * t.ldw);
    staged_product<T, T, true, !TRANSPOSED, BM, BN, WM, WN>((const T*)t.x + r0 * t.ldx, t.ldx, r1 - r0, w, t.ldw, (int)(t.out - n0), t.in,
                                                            (T*)t.y + r0 * t.ldy + n0, t.ldy);
}

template <typename T, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM* WN * 64) void product_grad_staged_kernel(HopProductGradTask t, int tiles_out, int tiles_in, HopIndex index) {
    int row, column;
    if (!place_tile(blockIdx.x, t.rows.G * tiles_out, tiles_in, &row, &column)) return;
    const int g = row / tiles_out;
    int b, e;
    group_rows(t.rows, g, &b, &e);
    const int64_t o0 = (int64_t)(row - g * tiles_out) * BM, i0 = (int64_t)column * BN;
    const int at = t.indexed ? index.at[g] : g;
    staged_product<T, float, false, false, BM, BN, WM, WN>((const T*)t.dy + b * t.lddy + o0, t.lddy, (int)(t.out - o0), (const T*)t.x + b * t.ldx + i0,
                                                           t.ldx, (int)(t.in - i0), e - b, t.dw + at * t.dw_stride + o0 * t.lddw + i0, t.lddw);
}

template <typename T, bool TRANSPOSED>
__global__ __launch_bounds__(kThreads) void product_kernel(HopProductTask t, HopIndex index) {
    int g, r0, r1;
    if (!find_piece(t.rows, 6, blockIdx.x, &g, &r0, &r1)) return;
    const int64_t n0 = (int64_t)blockIdx.y * kTile;
    const int at = t.indexed ? index.at[g] : g;
    const T* w = (const T*)t.w + at * t.w_stride + (TRANSPOSED ? n0 : n0 * t.ldw);
    tile_product<T, T, true, !TRANSPOSED>((const T*)t.x + r0 * t.ldx, t.ldx, r1 - r0, w, t.ldw, (int)(t.out - n0), t.in,
                                          (T*)t.y + r0 * t.ldy + n0, t.ldy);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void product_grad_kernel(HopProductGradTask t, HopIndex index) {
    const int g = blockIdx.z;
    int b, e;
    group_rows(t.rows, g, &b, &e);
    const int64_t o0 = (int64_t)blockIdx.y * kTile, i0 = (int64_t)blockIdx.x * kTile;
    const int at = t.indexed ? index.at[g] : g;
    tile_product<T, float, false, false>((const T*)t.dy + b * t.lddy + o0, t.lddy, (int)(t.out - o0), (const T*)t.x + b * t.ldx + i0, t.ldx,
                                         (int)(t.in - i0), e - b, t.dw + at * t.dw_stride + o0 * t.lddw + i0, t.lddw);
}

// Whether an operand can be fed by 128-bit loads: addresses and distances are multiples of 16 bytes, `cols` (the contiguous direction) of
// whole chunks, and a tile's offsets fit 31 bits.
bool feedable(const void* p, int64_t ld, int64_t stride, int64_t cols, size_t elem) {
    const int64_t chunk = 16 / (int64_t)elem;
    return ((uintptr_t)p & 15u) == 0 && ld % chunk == 0 && stride % chunk == 0 && cols % chunk == 0 && ld <= (1 << 20);
}

int64_t pieces_of(const HopRows& rows, int step) { return rows.rows / step + (rows.G < rows.rows ? rows.G : rows.rows); }

template <typename T, int BM, int BN, int WM, int WN>
bool launch_staged(const HopProductTask& t, int transposed, const HopIndex& index, hipStream_t st) {
    const int64_t columns = (t.out + BN - 1) / BN, tiles = pieces_of(t.rows, BM) * columns;
    if (tiles > 1 << 22) return false;
    const dim3 grid((unsigned)tiles), block(WM * WN * 64);
    if (transposed) product_staged_kernel<T, true, BM, BN, WM, WN><<<grid, block, 0, st>>>(t, (int)columns, index);
    else product_staged_kernel<T, false, BM, BN, WM, WN><<<grid, block, 0, st>>>(t, (int)columns, index);
    return true;
}

template <typename T>
bool staged(const HopProductTask& t, int transposed, const HopIndex& index, hipStream_t st) {
    if (!feedable(t.x, t.ldx, 0, t.in, sizeof(T)) || !feedable(t.w, t.ldw, t.w_stride, transposed ? t.out : t.in, sizeof(T))) return false;
    if constexpr (sizeof(T) == 2) return launch_staged<T, HOPL_BM, HOPL_BN, HOPL_WM, HOPL_WN>(t, transposed, index, st);
    else return launch_staged<T, 64, 128, 2, 2>(t, transposed, index, st);
}

template <typename T, int BM, int BN, int WM, int WN>
bool launch_grad_staged(const HopProductGradTask& t, const HopIndex& index, hipStream_t st) {
    const int64_t out = (t.out + BM - 1) / BM, in = (t.in + BN - 1) / BN, tiles = t.rows.G * out * in;
    if (tiles > 1 << 22) return false;
    product_grad_staged_kernel<T, BM, BN, WM, WN><<<dim3((unsigned)tiles), WM * WN * 64, 0, st>>>(t, (int)out, (int)in, index);
    return true;
}

template <typename T>
bool grad_staged(const HopProductGradTask& t, const HopIndex& index, hipStream_t st) {
    if (!feedable(t.dy, t.lddy, 0, t.out, sizeof(T)) || !feedable(t.x, t.ldx, 0, t.in, sizeof(T))) return false;
    if constexpr (sizeof(T) == 2) return launch_grad_staged<T, HOPL_BM, HOPL_BN, HOPL_WM, HOPL_WN>(t, index, st);
    else return launch_grad_staged<T, 128, 128, 2, 2>(t, index, st);
}

}  // namespace

int hopl_product(const HopProductTask& t, int dtype, int transposed, const HopIndex& index, void* stream) {
    hipStream_t st = (hipStream_t)stream;
    if (dtype == HOP_BF16 ? staged<bf16>(t, transposed, index, st) : staged<float>(t, transposed, index, st)) return (int)hipGetLastError();
    const dim3 grid((unsigned)pieces_of(t.rows, kTile), (unsigned)((t.out + kTile - 1) / kTile));
    if (dtype == HOP_BF16) {
        if (transposed) product_kernel<bf16, true><<<grid, kThreads, 0, st>>>(t, index);
        else product_kernel<bf16, false><<<grid, kThreads, 0, st>>>(t, index);
    } else {
        if (transposed) product_kernel<float, true><<<grid, kThreads, 0, st>>>(t, index);
        else product_kernel<float, false><<<grid, kThreads, 0, st>>>(t, index);
    }
    return (int)hipGetLastError();
}

int hopl_product_grad(const HopProductGradTask& t, int dtype, const HopIndex& index, void* stream) {
    hipStream_t st = (hipStream_t)stream;
    if (dtype == HOP_BF16 ? grad_staged<bf16>(t, index, st) : grad_staged<float>(t, index, st)) return (int)hipGetLastError();
    const dim3 grid((unsigned)((t.in + kTile - 1) / kTile), (unsigned)((t.out + kTile - 1) / kTile), (unsigned)t.rows.G);
    if (dtype == HOP_BF16) product_grad_kernel<bf16><<<grid, kThreads, 0, st>>>(t, index);
    else product_grad_kernel<float><<<grid, kThreads, 0, st>>>(t, index);
    return (int)hipGetLastError();
}
