// Products of rows grouped by worker or expert with their group's weights, and the gradient to the weights, for gfx950.
#include "hop_layers_device.h"

using namespace hopl;

namespace {

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

}  // namespace

int hopl_product(const HopProductTask& t, int dtype, int transposed, const HopIndex& index, void* stream) {
    hipStream_t st = (hipStream_t)stream;
    const int64_t pieces = t.rows.rows / kTile + (t.rows.G < t.rows.rows ? t.rows.G : t.rows.rows);
    const dim3 grid((unsigned)pieces, (unsigned)((t.out + kTile - 1) / kTile));
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
    const dim3 grid((unsigned)((t.in + kTile - 1) / kTile), (unsigned)((t.out + kTile - 1) / kTile), (unsigned)t.rows.G);
    if (dtype == HOP_BF16) product_grad_kernel<bf16><<<grid, kThreads, 0, st>>>(t, index);
    else product_grad_kernel<float><<<grid, kThreads, 0, st>>>(t, index);
    return (int)hipGetLastError();
}
