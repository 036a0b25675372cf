// Products of rows grouped by worker or expert with their group's weights, and the gradient to the weights, for gfx950 (CDNA4).
//
//   hop_product       y[r, n]    = sum_k x[r, k] w_g[n, k]   (transposed: w_g[k, n])      2 rows in out operations
//   hop_product_grad  dw_g[n, k] = sum_r dy[r, n] x[r, k]    over the group's rows        the same
//
// One kernel body computes c[p][q] = sum_k P(p, k) Q(q, k) by tiles on the matrix unit, for every combination of operands whose contraction
// is contiguous in memory or not, sums in fp32; what differs is where a tile's lines come from.  What bounds it: with about 200 rows a group or more the matrix unit
// (bf16: 8192^3 in 884 us, 1243 TFLOP/s; 16384 rows over 32 groups of 4096 x 4096 627 us, 877; fp32: 4096^3 in 978 us, 141 TFLOP/s, of 154 that
// a large library product reaches), with fewer the weights' bytes (128 rows over 64 groups of 4096 x 2048 in bf16: 184 us, 5.9 TB/s), in the gradient what it
// writes (the same groups: 326 us for 2.1 GB), and in small layers the launch.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "hop_layers_device.h"

using namespace hopl;

namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));

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

// ---- staged tiles -------------------------------------------------------------------
// Tiles of 128 bytes of the contraction, fed to LDS by the memory unit itself (128-bit loads that pass no register) into one of two
// stages while the matrix instructions run on the other.  An operand whose contraction is contiguous (ALONG) lies in LDS line by
// line, eight 16-byte chunks each; one whose lines are contiguous lies there row of the contraction by row.  The memory unit fills
// LDS in the order of the lanes, so what moves to keep the reads off each other's banks is which chunk a lane asks for: chunk c of
// line l stands at place c ^ (l / 2 mod 8); chunk c of row k at c ^ 4 (k mod 4) in 16 bits (c ^ 4 (k / 2 mod 2) where a row has
// only 8), c ^ 4 (k / 4 mod 4) in 32.  The loads go through a buffer descriptor whose end is the operand's: what lies outside comes back as zero.
constexpr int kStepBytes = 128;
constexpr uint32_t kOutside = 0x80000000u;      // beyond any descriptor's end

template <typename T, int LINES>
__device__ __forceinline__ int across_swizzle(int k) {
    if (sizeof(T) == 4) return ((k >> 2) & 3) << 2;
    return LINES >= 128 ? (k & 3) << 2 : ((k >> 1) & 1) << 2;
}

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

    static __device__ __forceinline__ int swizzle(int l) { return ALONG ? (l >> 1) & 7 : across_swizzle<T, LINES>(l); }
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

// The same for operands of any alignment, through registers: 128-bit loads at an element's address, chunks cut where the operand ends.
template <typename T, bool ALONG, int LINES, int NT>
struct RegisterFeed {
    static constexpr int kChunk = 16 / sizeof(T), kK = kStepBytes / sizeof(T), kPerLine = ALONG ? 8 : LINES / kChunk, kLoads = LINES * 8 / NT;
    static constexpr int kBytes = LINES * kStepBytes;
    typedef T chunk __attribute__((ext_vector_type(kChunk)));
    typedef chunk chunk_any __attribute__((aligned(sizeof(T))));
    const T* base;
    int64_t ld;
    int lines, K;
    chunk part[kLoads];

    __device__ __forceinline__ void start(const T* p, int64_t ld_, int lines_, int K_) {
        base = p;
        ld = ld_;
        lines = lines_ < LINES ? lines_ : LINES;
        K = K_;
    }
    // Chunks that begin inside the operand are loaded whole wherever that stays in front of its last element.  What they hold beyond the
    // contraction's end is set to zero on the way to LDS (not here: the loads are to be on their way through a turn); beyond the last line
    // they fill lines whose results nobody stores.
    __device__ __forceinline__ void fetch(int k) {
        const int64_t end = ALONG ? (lines - 1) * ld + K : (K - 1) * ld + lines;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int j = i * NT + threadIdx.x, l = j / kPerLine, c = j % kPerLine * kChunk;
            const int n = ALONG ? (l < lines ? K - k - c : 0) : (k + l < K ? lines - c : 0);
            const int64_t off = ALONG ? l * ld + (k + c) : (int64_t)(k + l) * ld + c;
            part[i] = (T)0.f;
            if (n <= 0) continue;
            const HOPL_GLOBAL T* p = (const HOPL_GLOBAL T*)(base + off);
            if (off + kChunk <= end) {
                part[i] = *(const HOPL_GLOBAL chunk_any*)p;
            } else {
                part[i] = load_short<chunk>(base + off, n < kChunk ? n : kChunk);
            }
        }
    }
    __device__ __forceinline__ void put(char* stage, int k) {
        if (ALONG && K - k < kK) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int n = K - k - (i * NT + (int)threadIdx.x) % kPerLine * kChunk;
#pragma unroll
                for (int e = 0; e < kChunk; ++e)
                    if (e >= n) part[i][e] = (T)0.f;
            }
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int j = i * NT + threadIdx.x, l = j / kPerLine, c = (j % kPerLine) ^ Feed<T, ALONG, LINES, NT>::swizzle(l);
            *(chunk*)(stage + (l * kPerLine + c) * 16) = part[i];
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
        const int k = turn * 16 + (lane >> 5) * 8 + row, place = (((line >> 3) ^ across_swizzle<bf16, LINES>(row)) << 4) + (line & 4) * 2;
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
        const char* at = s + (turn * 16 + quad * 4) * LINES * 4 + ((((line >> 2) ^ across_swizzle<float, LINES>(quad * 4)) << 4) + (line & 3) * 4);
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

template <typename T, typename OUT, bool PA, bool QA, bool FED, int BM, int BN, int WM, int WN>
__device__ __forceinline__ void staged_product(const T* p, int64_t ldp, int np, const T* q, int64_t ldq, int nq, int K, OUT* c, int64_t ldc) {
    typedef Unit<T> U;
    constexpr int NT = WM * WN * 64, TM = BM / WM, TN = BN / WN, FM = TM / U::kLines, FN = TN / U::kLines;
    constexpr int kK = kStepBytes / sizeof(T);
    // Which operand comes first decides what a lane holds of the result: four consecutive columns of a row, or four rows of a column.
    // For results in 32 bits of a 32-line unit the latter: 32 lanes store 128 consecutive bytes of a row.
    constexpr bool kSwap = sizeof(OUT) == 4 && U::kLines == 32;
    typedef std::conditional_t<FED, Feed<T, PA, BM, NT>, RegisterFeed<T, PA, BM, NT>> P;
    typedef std::conditional_t<FED, Feed<T, QA, BN, NT>, RegisterFeed<T, QA, BN, NT>> Q;
    // arrays of their own, so that the compiler knows that reads of one stage need not wait for loads into the other
    __shared__ __attribute__((aligned(16))) char sp0[P::kBytes], sq0[Q::kBytes], sp1[P::kBytes], sq1[Q::kBytes];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    // A wavefront's units of rows lie WM apart, so that a piece of few rows leaves each of them as few, and `live` of them are multiplied.
    const int p0 = (wave % WM) * U::kLines, q0 = (wave / WM) * TN;
    constexpr int kNext = WM * U::kLines;
    typename U::acc acc[FN][FM] = {};
    P fp;
    Q fq;
    fp.start(p, ldp, np, K);
    fq.start(q, ldq, nq, K);
    // Tiles of few rows are bound by reading the other operand, whose lines are a power of two apart as a rule: workgroups that walk along
    // them side by side would all ask the same memory channels.  So they begin at different places and go round.
    const int steps = (K + kK - 1) / kK, rotate = np <= kNext && steps ? (int)(blockIdx.x / 8 % steps) : 0;
    auto begins = [&](int step) { return (step + rotate < steps ? step + rotate : step + rotate - steps) * kK; };
    auto issue = [&](char* sp, char* sq, int step) {
        const int k = begins(step);
        if constexpr (FED) {
            fp.issue(sp, k);
            fq.issue(sq, k);
        } else {
            fp.fetch(k);
            fq.fetch(k);
        }
    };
    auto put = [&](char* sp, char* sq, int step) {            // behind the turn that the loads ran beside
        if constexpr (!FED) {
            const int k = begins(step);
            fp.put(sp, k);
            fq.put(sq, k);
        }
    };
    if (steps) {
        issue(sp0, sq0, 0);
        put(sp0, sq0, 0);
    }
    auto run = [&](auto live) {
        constexpr int kLive = decltype(live)::value;
        auto turn = [&](const char* sp, const char* sq) {
#pragma unroll
            for (int t = 0; t < U::kTurns; ++t) {
                typename U::frag a[kLive], b[FN];
#pragma unroll
                for (int i = 0; i < FN; ++i) {
                    if constexpr (QA) b[i] = U::along(sq, q0 + U::kLines * i, t);
                    else b[i] = U::template across<BN>(sq, q0 + U::kLines * i, t);
                }
#pragma unroll
                for (int j = 0; j < kLive; ++j) {
                    if constexpr (PA) a[j] = U::along(sp, p0 + kNext * j, t);
                    else a[j] = U::template across<BM>(sp, p0 + kNext * j, t);
                }
#pragma unroll
                for (int j = 0; j < kLive; ++j)
#pragma unroll
                    for (int i = 0; i < FN; ++i) acc[i][j] = kSwap ? U::step(a[j], b[i], acc[i][j]) : U::step(b[i], a[j], acc[i][j]);
                if (t & 1) __builtin_amdgcn_sched_barrier(0);      // fragments of two turns at a time: all at once do not fit the registers
            }
        };
        int step = 0;
        for (; step + 1 < steps; step += 2) {
            arrive();
            issue(sp1, sq1, step + 1);
            turn(sp0, sq0);
            put(sp1, sq1, step + 1);
            arrive();
            if (step + 2 < steps) issue(sp0, sq0, step + 2);
            turn(sp1, sq1);
            if (step + 2 < steps) put(sp0, sq0, step + 2);
        }
        if (step < steps) {
            arrive();
            turn(sp0, sq0);
        }
    };
    const int live = (np + kNext - 1) / kNext;
    if (FM == 1 || live >= FM) run(std::integral_constant<int, FM>());
    else if (FM > 2 && live == 3) run(std::integral_constant<int, FM < 3 ? FM : 3>());
    else if (FM > 1 && live == 2) run(std::integral_constant<int, FM < 2 ? FM : 2>());
    else run(std::integral_constant<int, 1>());
    constexpr int kQuads = sizeof(typename U::acc) / 16;
    if constexpr (kSwap) {
#pragma unroll
        for (int j = 0; j < FM; ++j)
#pragma unroll
            for (int v = 0; v < 4 * kQuads; ++v) {
                const int row = p0 + kNext * j + U::column(v >> 2) + (v & 3);
                if (row >= np) continue;
                OUT* to = c + row * ldc + q0 + (lane & (U::kLines - 1));
#pragma unroll
                for (int i = 0; i < FN; ++i)
                    if (q0 + U::kLines * i + (lane & (U::kLines - 1)) < nq) ((HOPL_GLOBAL OUT*)to)[U::kLines * i] = acc[i][j][v];
            }
        return;
    }
#pragma unroll
    for (int j = 0; j < FM; ++j) {
        const int row = p0 + kNext * j + (lane & (U::kLines - 1));
        if (row >= np) continue;
        OUT* to = c + row * ldc;
#pragma unroll
        for (int i = 0; i < FN; ++i)
#pragma unroll
            for (int v = 0; v < kQuads; ++v) {
                const int col = q0 + U::kLines * i + U::column(v);
                if (col < nq) store4(to + col, nq - col, f32x4{acc[i][j][4 * v], acc[i][j][4 * v + 1], acc[i][j][4 * v + 2], acc[i][j][4 * v + 3]});
            }
    }
}

// Which tile a workgroup takes.  Workgroups are dealt to the 8 XCDs in turn; an XCD takes runs of up to 32 tiles (a workgroup for each of its CUs),
// kBand pieces of rows by 8 columns of tiles, so that both operands' tiles are found in its L2 again, and the runs go round the XCDs, so
// that each gets its share of whole and of short pieces.  `most` is the number of workgroups for all tiles that there can be: a launch may hold
// a part of them only, from workgroup `first` on.
constexpr int kBand = 4, kRun = 32;
__device__ __forceinline__ bool place_tile(int b, int most, int pieces, int columns, int* piece, int* column) {
    pieces = min(pieces, most / columns);                   // what a proper row table has at most
    const int total = pieces * columns, rounds = (total + 8 * kRun - 1) / (8 * kRun);
    if (!total) return false;
    const int run = (total + 8 * rounds - 1) / (8 * rounds), turn = b / 8;      // as many runs for every XCD
    const int at = (turn / run * 8 + b % 8) * run + turn % run;
    if (at >= total) return false;
    const int band = at / (kBand * columns), within = at - band * kBand * columns;
    const int height = pieces - band * kBand < kBand ? pieces - band * kBand : kBand;
    *column = within / height;
    *piece = band * kBand + within % height;
    return true;
}

// PART: the contraction is cut in gridDim.y parts, whose sums go to partial[part][row][column] in 32 bits.
template <typename T, bool TRANSPOSED, bool PART, bool FED, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM* WN * 64) void product_staged_kernel(HopProductTask t, int columns, int first, int most, HopIndex index) {
    constexpr int shift = __builtin_ctz(BM), kK = kStepBytes / sizeof(T);
    int piece, column, g, r0, r1;
    if constexpr (BM >= 256) {
        const WholePieces all = count_whole(t.rows, shift);
        if (!place_tile(first + blockIdx.x, most, all.whole + all.rest, columns, &piece, &column) || !find_whole(t.rows, shift, all, piece, &g, &r0, &r1)) return;
    } else {                    // a group's pieces together: they share its weights
        if (!place_tile(first + blockIdx.x, most, count_pieces(t.rows, shift), columns, &piece, &column) || !find_piece(t.rows, shift, piece, &g, &r0, &r1)) return;
    }
    const int64_t n0 = (int64_t)column * BN;
    const int at = t.indexed ? index.at[g] : g;
    const T* x = (const T*)t.x + r0 * t.ldx;
    const T* w = (const T*)t.w + at * t.w_stride + (TRANSPOSED ? n0 : n0 * t.ldw);
    if constexpr (PART) {
        const int each = ((t.in + gridDim.y - 1) / gridDim.y + kK - 1) / kK * kK, k0 = min((int)blockIdx.y * each, t.in);
        staged_product<T, float, true, !TRANSPOSED, FED, BM, BN, WM, WN>(x + k0, t.ldx, r1 - r0, w + (TRANSPOSED ? k0 * t.ldw : k0), t.ldw, (int)(t.out - n0),
                                                                    min(each, t.in - k0),
                                                                    t.partial + ((int64_t)blockIdx.y * t.rows.rows + r0) * t.out + n0, t.out);
    } else {
        staged_product<T, T, true, !TRANSPOSED, FED, BM, BN, WM, WN>(x, t.ldx, r1 - r0, w, t.ldw, (int)(t.out - n0), t.in, (T*)t.y + r0 * t.ldy + n0, t.ldy);
    }
}

// PART: the group's rows are cut in gridDim.y parts, whose sums go to partial[part][g][out][in].
template <typename T, bool PART, bool FED, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM* WN * 64) void product_grad_staged_kernel(HopProductGradTask t, int tiles_out, int tiles_in, int first, HopIndex index) {
    constexpr int kK = kStepBytes / sizeof(T);
    // Groups differ in length, so every group's tiles are dealt to all XCDs, a run of them to each (operands' tiles are shared in its L2).
    const int tiles = tiles_out * tiles_in, each_xcd = (tiles + 7) / 8, x = blockIdx.x % 8, turn = (first + (int)blockIdx.x) / 8;
    const int g = turn / each_xcd, tile = x * each_xcd + turn % each_xcd;
    if (tile >= tiles) return;
    const int row = tile / tiles_in, column = tile % tiles_in;
    int b, e;
    group_rows(t.rows, g, &b, &e);
    const int64_t o0 = (int64_t)row * BM, i0 = (int64_t)column * BN;
    float* to = t.dw + (t.indexed ? index.at[g] : g) * t.dw_stride + o0 * t.lddw + i0;
    int64_t ld = t.lddw;
    if (PART) {
        const int each = ((e - b + (int)gridDim.y - 1) / (int)gridDim.y + kK - 1) / kK * kK;
        b = min(b + (int)blockIdx.y * each, e);
        e = min(b + each, e);
        to = t.partial + (((int64_t)blockIdx.y * t.rows.G + g) * t.out + o0) * t.in + i0;
        ld = t.in;
    }
    staged_product<T, float, false, false, FED, BM, BN, WM, WN>((const T*)t.dy + b * t.lddy + o0, t.lddy, (int)(t.out - o0), (const T*)t.x + b * t.ldx + i0,
                                                           t.ldx, (int)(t.in - i0), e - b, to, ld);
}

// The parts' sums of eight columns, in order: y for hop_product, dw for its gradient (a row is (group, out) there).
template <typename OUT>
__global__ __launch_bounds__(256) void product_join_kernel(const float* partial, int parts, int64_t rows, int cols, OUT* to, int64_t ld, int per_group,
                                                           int64_t group_stride, int indexed, HopIndex index) {
    const int chunks = (cols + 7) / 8;
    const int64_t all = rows * chunks, one = rows * cols;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / chunks;
        const int c = (int)(i - r * chunks) * 8;
        const float* from = partial + r * cols + c;
        f32x8 a = load8(from, cols - c);
#pragma unroll 4
        for (int p = 1; p < parts; ++p) a += load8(from + p * one, cols - c);
        const int64_t g = per_group ? r / per_group : 0;
        OUT* out = per_group ? to + (indexed ? index.at[g] : g) * group_stride + (r - g * per_group) * ld : to + r * ld;
        store8(out + c, cols - c, a);
    }
}
inline unsigned join_blocks(int64_t rows, int cols) {
    const int64_t n = (rows * ((cols + 7) / 8) + 255) / 256;
    return (unsigned)(n < 4096 ? n : 4096);
}

// ---- few rows -----------------------------------------------------------------------
// 16 FM rows by 16 columns: the weights are read once, straight into the registers that the matrix unit takes them from (a lane holds 32
// consecutive bytes of its line, four lanes a cache line), by four wavefronts that take turns along the contraction and join their
// sums in LDS.  Bound by reading the weights; a tile's share of them is a few KB, so that small layers have workgroups for every CU.  Of a pass's
// 16 to 24 loads a wavefront, 16 rows in bf16 have eight on their way as the compiler orders them, 32 rows five to seven (over 16 wavefronts four),
// fp32 four.
template <typename T, int FM, int kFewWaves>
__global__ __launch_bounds__(kFewWaves * 64) void product_few_kernel(HopProductTask t, HopIndex index) {
    constexpr int kChunk = 16 / sizeof(T), kK = 8 * kChunk, kUnroll = 4;      // elements of a load, of a turn; turns a pass of the loop
    __shared__ f32x4 s[kFewWaves][FM][64];
    int g, r0, r1;
    if (!find_piece(t.rows, 4 + (FM >> 1), blockIdx.y, &g, &r0, &r1)) return;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, l16 = lane & 15, quad = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * 16;
    const int columns = (int)min((int64_t)16, t.out - n0), K = t.in;
    const int at = t.indexed ? index.at[g] : g;
    const T* w = (const T*)t.w + at * t.w_stride + n0 * t.ldw;
    const T* x = (const T*)t.x + r0 * t.ldx;
    const __amdgpu_buffer_rsrc_t rw = __builtin_amdgcn_make_buffer_rsrc((void*)w, 0, (int)(((columns - 1) * t.ldw + K) * sizeof(T)), 0x00020000);
    const __amdgpu_buffer_rsrc_t rx = __builtin_amdgcn_make_buffer_rsrc((void*)x, 0, (int)(((r1 - r0 - 1) * t.ldx + K) * sizeof(T)), 0x00020000);
    const uint32_t ow = (uint32_t)(l16 * t.ldw * sizeof(T)), ox = (uint32_t)(l16 * t.ldx * sizeof(T)), next = (uint32_t)(16 * t.ldx * sizeof(T));
    f32x4 acc[FM] = {};
    typedef std::conditional_t<sizeof(T) == 2, bf16x8, f32x4> frag;
    union raw { u32x4 u; frag f; };
#pragma unroll 1
    for (int k0 = wave * kK; k0 < K; k0 += kFewWaves * kK * kUnroll) {
        raw a[kUnroll][FM][2], b[kUnroll][2];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = k0 + u * kFewWaves * kK + (quad * 2 + h) * kChunk;
                const uint32_t o = (uint32_t)k * sizeof(T);
                b[u][h].u = __builtin_amdgcn_raw_buffer_load_b128(rw, k < K && l16 < columns ? ow + o : kOutside, 0, 0);
#pragma unroll
                for (int j = 0; j < FM; ++j)
                    a[u][j][h].u = __builtin_amdgcn_raw_buffer_load_b128(rx, k < K && l16 + 16 * j < r1 - r0 ? ox + j * next + o : kOutside, 0, 0);
            }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < FM; ++j) {
                    if constexpr (sizeof(T) == 2) {
                        acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[u][h].f, a[u][j][h].f, acc[j], 0, 0, 0);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(b[u][h].f[e], a[u][j][h].f[e], acc[j], 0, 0, 0);
                    }
                }
    }
#pragma unroll
    for (int j = 0; j < FM; ++j) s[wave][j][lane] = acc[j];
    __syncthreads();
    if (wave >= FM) return;
    f32x4 v = s[0][wave][lane];
#pragma unroll
    for (int i = 1; i < kFewWaves; ++i) v += s[i][wave][lane];
    const int row = wave * 16 + l16, col = quad * 4;
    if (row < r1 - r0 && col < columns) store4((T*)t.y + (r0 + row) * t.ldy + n0 + col, columns - col, v);
}

// Whether an operand can be fed by 128-bit loads: addresses and distances are multiples of 16 bytes, `cols` (the contiguous direction) of
// whole chunks, and a tile's offsets fit 31 bits.
bool feedable(const void* p, int64_t ld, int64_t stride, int64_t cols, size_t elem) {
    const int64_t chunk = 16 / (int64_t)elem;
    return ((uintptr_t)p & 15u) == 0 && ld % chunk == 0 && stride % chunk == 0 && cols % chunk == 0 && ld <= (1 << 20);
}

// The most pieces of `step` rows that G groups can leave: each group with rows has at most step - 1 of them missing from its last.
int64_t pieces_of(const HopRows& rows, int step) { return (rows.rows + (int64_t)(step - 1) * (rows.G < rows.rows ? rows.G : rows.rows)) / step; }
// Workgroups that place_tile needs to see them all.
int64_t tile_grid(int64_t tiles) { return 8 * ((tiles + 7) / 8 + (tiles + 8 * kRun - 1) / (8 * kRun)); }

// A launch holds fewer than 2^32 threads.  More workgroups than these go in several (parts of a multiple of 8, so that XCDs get what they would).
constexpr int64_t kMostBlocks = 1 << 22;
template <typename F>
void in_launches(int64_t blocks, F launch) {
    for (int64_t first = 0; first < blocks; first += kMostBlocks) launch((int)first, (unsigned)std::min(kMostBlocks, blocks - first));
}

template <typename T, bool FED, int BM, int BN, int WM, int WN>
void launch_staged(const HopProductTask& t, int transposed, int parts, const HopIndex& index, hipStream_t st) {
    const int64_t columns = (t.out + BN - 1) / BN, most = tile_grid(pieces_of(t.rows, BM) * columns);
    in_launches(most, [&](int first, unsigned blocks) {
        const dim3 grid(blocks, (unsigned)parts), block(WM * WN * 64);
        if (parts > 1 && transposed) product_staged_kernel<T, true, true, FED, BM, BN, WM, WN><<<grid, block, 0, st>>>(t, (int)columns, first, (int)most, index);
        else if (parts > 1) product_staged_kernel<T, false, true, FED, BM, BN, WM, WN><<<grid, block, 0, st>>>(t, (int)columns, first, (int)most, index);
        else if (transposed) product_staged_kernel<T, true, false, FED, BM, BN, WM, WN><<<grid, block, 0, st>>>(t, (int)columns, first, (int)most, index);
        else product_staged_kernel<T, false, false, FED, BM, BN, WM, WN><<<grid, block, 0, st>>>(t, (int)columns, first, (int)most, index);
    });
    if (parts > 1)
        product_join_kernel<T><<<join_blocks(t.rows.rows, t.out), 256, 0, st>>>(t.partial, parts, t.rows.rows, t.out, (T*)t.y, t.ldy, 0, 0, 0, index);
}
template <typename T, bool FED>
void launch_tile(const HopProductTask& t, int transposed, const HopProductPlan& p, const HopIndex& index, hipStream_t st) {
    if (p.tile == 1) launch_staged<T, FED, 128, 128, 2, 2>(t, transposed, p.parts, index, st);
    else if (p.tile == 2) launch_staged<T, FED, 64, 64, 2, 2>(t, transposed, p.parts, index, st);
    else launch_staged<T, FED, 32, 128, 1, 4>(t, transposed, p.parts, index, st);
}

template <typename T>
void launch_few(const HopProductTask& t, int tile, const HopIndex& index, hipStream_t st) {
    const dim3 grid((unsigned)((t.out + 15) / 16), (unsigned)pieces_of(t.rows, tile & 1 ? 32 : 16));
    if (tile == 0) product_few_kernel<T, 1, 4><<<grid, 256, 0, st>>>(t, index);
    else if (tile == 1) product_few_kernel<T, 2, 4><<<grid, 256, 0, st>>>(t, index);
    else if (tile == 2) product_few_kernel<T, 1, 16><<<grid, 1024, 0, st>>>(t, index);
    else product_few_kernel<T, 2, 16><<<grid, 1024, 0, st>>>(t, index);
}

// Gradients in 32 bits on 128 x 128 tiles are not cut in parts: 64 x 64 tiles take 0.99 of the time a step and have the grain of four parts with
// nothing to join, so the estimate never came out that way (1.6 million sizes).
template <typename T, int BM>
constexpr bool kInParts = sizeof(T) == 2 || BM < 128;

template <typename T, bool FED, int BM, int BN, int WM, int WN>
void launch_grad_staged(const HopProductGradTask& t, int parts, const HopIndex& index, hipStream_t st) {
    const int64_t out = (t.out + BM - 1) / BM, in = (t.in + BN - 1) / BN;
    in_launches(t.rows.G * ((out * in + 7) / 8 * 8), [&](int first, unsigned blocks) {
        const dim3 grid(blocks, (unsigned)parts), block(WM * WN * 64);
        if constexpr (kInParts<T, BM>) {
            if (parts > 1) return product_grad_staged_kernel<T, true, FED, BM, BN, WM, WN><<<grid, block, 0, st>>>(t, (int)out, (int)in, first, index);
        }
        product_grad_staged_kernel<T, false, FED, BM, BN, WM, WN><<<grid, block, 0, st>>>(t, (int)out, (int)in, first, index);
    });
    if (parts > 1) {
        const int64_t rows = (int64_t)t.rows.G * t.out;
        product_join_kernel<float><<<join_blocks(rows, t.in), 256, 0, st>>>(t.partial, parts, rows, t.in, t.dw, t.lddw, t.out, t.dw_stride, t.indexed, index);
    }
}

// ---- which way ----------------------------------------------------------------------
// Tiles and parts are chosen by an estimate of each way's time from the sizes; how the rows fall to the groups is not known here, so
// groups are taken for equal.  The constants are measured (MI355X, us): `full`, a step of 128 bytes of the contraction on a CU that
// has enough workgroups (bf16 256 x 256: 8192^3 in 884 us; fp32 128 x 128: 4096^3 in 978); `least`, of a workgroup that has the CU to itself, bound
// by the loads' latency; `beside`, workgroups that a CU holds; `own`, what a workgroup costs beside its steps (told apart for gradients only).
struct TileCost {
    int bm, bn, grain;             // rows and columns; rows that a short piece is rounded up to
    double full, least;
    int beside;
    double own = 0.0;
};
constexpr TileCost kTilesBf16[4] = {{256, 256, 64, 1.75, 0.85, 1}, {128, 128, 64, 0.49, 0.55, 2}, {64, 64, 64, 0.24, 0.45, 5}, {32, 128, 32, 0.28, 0.46, 4}};
constexpr TileCost kTilesF32[4] = {{0, 0, 0, 0, 0, 0}, {128, 128, 32, 1.91, 0.75, 2}, {64, 64, 32, 0.49, 0.62, 5}, {32, 128, 16, 0.50, 0.60, 4}};
constexpr TileCost kGradTilesBf16[3] = {{256, 256, 64, 1.75, 1.1, 1}, {128, 128, 64, 0.60, 0.67, 2, 0.5}, {64, 64, 64, 0.35, 0.45, 4, 0.3}};
constexpr TileCost kGradTilesF32[2] = {{128, 128, 32, 1.93, 2.1, 2}, {64, 64, 32, 0.48, 0.65, 4, 0.2}};
constexpr double kCus = 256, kHbm = 5.2e6, kJoin = 6e6, kLaunch = 4;       // bytes a us; us

// Steps of `units` workgroups; `fill`: the part of a tile that is not padding; `far`: the weights are too many for the caches, which the
// smaller tiles feel (2048 rows over 16 groups of 1024 x 4096 in bf16, transposed: 1.0 us a step of 128 x 128, 0.55 from the L2).
double steps_time(const TileCost& c, double units, double steps, double fill, bool far) {
    const double each = std::max(1.0, std::ceil(units / kCus));
    const double one = std::max(c.least * (far && c.beside > 1 ? 1.6 : 1.0), c.beside == 1 ? c.full * fill : 1.1 * c.full * fill);
    return steps * std::max(std::ceil(each / c.beside) * one, each * c.full * fill) + each * c.own;
}

// Two things that run side by side, and get in each other's way a little.
double together(double a, double b) { return std::max(a, b) + 0.1 * std::min(a, b); }

}  // namespace

HopProductPlan hopl_product_plan(const HopProductTask& t, int dtype, int transposed) {
    HopProductPlan best = {HOPL_ANY, 1, 1};
    const size_t e = dtype == HOP_BF16 ? 2 : 4;
    const bool fed = feedable(t.x, t.ldx, 0, t.in, e) && feedable(t.w, t.ldw, t.w_stride, transposed ? t.out : t.in, e);
    const double T = t.rows.rows, G = std::min((double)t.rows.G, T), R = T / G, in = t.in, out = t.out;
    const double bytes = e * (G * in * out + T * in + T * out) / kHbm;
    double least = 1e300;
    auto consider = [&](double us, HopProductPlan p) {
        if (us < least) least = us, best = p;
    };
    for (int i = fed && dtype == HOP_BF16 ? 0 : 1; i < 4; ++i) {
        TileCost c = dtype == HOP_BF16 ? kTilesBf16[i] : kTilesF32[i];
        if (!fed) c.full *= 1.2, c.least *= 1.4;       // through registers (4096 x 4096 x 4095 in fp32: 1166 us, 994 when fed)
        if (dtype == HOP_F32 && transposed && i == 2) c.full *= 1.15;          // its reads of single words from LDS (4096^3: 1157 us, 1000 the other way)
        const double per = R <= c.bm / 2 ? 1 : R / c.bm + 0.5, fill = std::min(1.0, (R + c.grain / 2) / (per * c.bm));
        const double units = G * per * std::ceil(out / c.bn), steps = std::ceil(in * e / kStepBytes);
        for (int parts = 1; parts <= 8; parts *= 2) {
            if (parts > 1 && (steps < 2 * parts || units * parts > 10 * kCus)) break;
            double us = kLaunch + together(bytes, steps_time(c, units * parts, std::ceil(steps / parts), fill, G * in * out * e > 64e6));
            if (parts > 1) us += 3 + parts * T * out * 8 / kJoin;
            consider(us, {fed ? HOPL_FED : HOPL_ANY, parts, i});
        }
    }
    // Few rows: a turn of all wavefronts takes 1.25 us when nothing else is in its way; the kernel of 32 rows, with fewer loads on their way, reads
    // the weights at 3 TB/s (64 rows of 4096 x 4096 in bf16 26 us), that of 16 at 5 (33 us).  Sixteen wavefronts where there are too few workgroups for four of them each (1 row, 8192 x 1024:
    // 14.2 -> 12.7 us; 8 rows over 8 groups of 1024 x 1024 6.6 -> 9.6).
    if (fed && !transposed && R <= 128 && T * in * out < 1e12) {
        for (int wide = 0; wide < 2; ++wide) {
            const double pieces = G * std::max(1.0, R <= (wide ? 32 : 16) ? 1.0 : R / (wide ? 32 : 16) + 0.5), units = pieces * std::ceil(out / 16);
            const double turns = std::ceil(in * e / 2048.0);
            const bool many = units <= kCus && turns >= 4;
            const double us = kLaunch + together(bytes, std::max((many ? std::ceil(turns / 4) + 2 : turns) * 1.25, pieces * in * out * e / (wide ? 3.0e6 : 5.0e6)));
            consider(us, {HOPL_FEW, 1, wide + (many ? 2 : 0)});
        }
    }
    return best;
}

HopProductPlan hopl_product_grad_plan(const HopProductGradTask& t, int dtype) {
    HopProductPlan best = {HOPL_ANY, 1, dtype == HOP_BF16 ? 1 : 0};
    const size_t e = dtype == HOP_BF16 ? 2 : 4;
    const bool fed = feedable(t.dy, t.lddy, 0, t.out, e) && feedable(t.x, t.ldx, 0, t.in, e);
    const double G = t.rows.G, R = std::max(1.0, t.rows.rows / G), written = G * t.in * t.out * 4.0;
    double least = 1e300;
    for (int i = fed || dtype != HOP_BF16 ? 0 : 1; i < (dtype == HOP_BF16 ? 3 : 2); ++i) {
        const TileCost& c = dtype == HOP_BF16 ? kGradTilesBf16[i] : kGradTilesF32[i];
        const bool cut = dtype == HOP_BF16 || i > 0;             // kInParts
        const double units = G * std::ceil((double)t.out / c.bm) * std::ceil((double)t.in / c.bn), steps = std::ceil(R * e / kStepBytes);
        for (int parts = 1; parts <= 8; parts *= 2) {
            if (parts > 1 && (!cut || steps < 2 * parts || units * parts > 10 * kCus)) break;
            double us = kLaunch + 1.5 * (2 - i) + written / kHbm + steps_time(c, units * parts, std::ceil(steps / parts), 1.0, false);
            if (parts > 1) us += 3 + 2 * parts * written / kHbm;
            if (us < least) least = us, best = {fed ? HOPL_FED : HOPL_ANY, parts, i};
        }
    }
    return best;
}

int hopl_product(const HopProductTask& t, const HopProductPlan& p, int dtype, int transposed, const HopIndex& index, void* stream) {
    hipStream_t st = (hipStream_t)stream;
    if (p.kind == HOPL_FEW) {
        if (dtype == HOP_BF16) launch_few<bf16>(t, p.tile, index, st);
        else launch_few<float>(t, p.tile, index, st);
    } else if (dtype == HOP_BF16) {
        if (p.tile == 0) launch_staged<bf16, true, 256, 256, 2, 4>(t, transposed, p.parts, index, st);
        else if (p.kind == HOPL_FED) launch_tile<bf16, true>(t, transposed, p, index, st);
        else launch_tile<bf16, false>(t, transposed, p, index, st);
    } else {
        if (p.kind == HOPL_FED) launch_tile<float, true>(t, transposed, p, index, st);
        else launch_tile<float, false>(t, transposed, p, index, st);
    }
    return (int)hipGetLastError();
}

int hopl_product_grad(const HopProductGradTask& t, const HopProductPlan& p, int dtype, const HopIndex& index, void* stream) {
    hipStream_t st = (hipStream_t)stream;
    if (dtype == HOP_BF16) {
        if (p.tile == 0) launch_grad_staged<bf16, true, 256, 256, 2, 4>(t, p.parts, index, st);
        else if (p.kind == HOPL_FED && p.tile == 1) launch_grad_staged<bf16, true, 128, 128, 2, 2>(t, p.parts, index, st);
        else if (p.kind == HOPL_FED) launch_grad_staged<bf16, true, 64, 64, 2, 2>(t, p.parts, index, st);
        else if (p.tile == 1) launch_grad_staged<bf16, false, 128, 128, 2, 2>(t, p.parts, index, st);
        else launch_grad_staged<bf16, false, 64, 64, 2, 2>(t, p.parts, index, st);
    } else {
        if (p.kind == HOPL_FED && p.tile == 0) launch_grad_staged<float, true, 128, 128, 2, 2>(t, p.parts, index, st);
        else if (p.kind == HOPL_FED) launch_grad_staged<float, true, 64, 64, 2, 2>(t, p.parts, index, st);
        else if (p.tile == 0) launch_grad_staged<float, false, 128, 128, 2, 2>(t, p.parts, index, st);
        else launch_grad_staged<float, false, 64, 64, 2, 2>(t, p.parts, index, st);
    }
    return (int)hipGetLastError();
}
