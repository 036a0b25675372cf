// Norms before and after a block fused with its gate, dropout and residual sum, their gradients, and dropout by itself, for gfx950.
//
// About ten operations an element, so bytes bound all of it: a row is read once, stays in registers through its statistics
// (eight consecutive columns a thread and turn), and is written once; the mask is worked out again wherever it is needed.
#include <type_traits>

#include "hop_layers_device.h"

using namespace hopl;

namespace {

// ---- Philox4x32-10 ------------------------------------------------------------------
// Eight 16-bit draws of the counter (column / 8, row low, row high, 0).  Per round two 32 x 32 -> 64 bit products: about 170
// issue cycles per 64 x 8 elements, a third of what reading and writing them in 16 bits takes.
__device__ __forceinline__ void philox(const HopMask& m, uint32_t block, int64_t row, uint32_t (&out)[4]) {
    uint32_t c0 = block, c1 = (uint32_t)row, c2 = (uint32_t)((uint64_t)row >> 32), c3 = 0, k0 = m.k0, k1 = m.k1;
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    out[0] = c0; out[1] = c1; out[2] = c2; out[3] = c3;
}
// v where the mask keeps it, times its factor; 0 where not, whatever v is there.
__device__ __forceinline__ f32x8 dropped(const HopMask& m, uint32_t block, int64_t row, f32x8 v) {
    uint32_t w[4];
    philox(m, block, row, w);
    f32x8 r;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t draw = i & 1 ? w[i >> 1] >> 16 : w[i >> 1] & 0xFFFFu;
        r[i] = draw >= m.threshold ? v[i] * m.factor : 0.f;
    }
    return r;
}

template <typename T>
__global__ __launch_bounds__(256) void dropout_kernel(const T* x, int64_t ldx, T* y, int64_t ldy, int64_t rows, int64_t cols, HopMask m) {
    const int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (c >= cols) return;
    const int n = cols - c < 8 ? (int)(cols - c) : 8;
    for (int64_t r = blockIdx.y; r < rows; r += gridDim.y)
        store8(y + r * ldy + c, n, dropped(m, (uint32_t)(c >> 3), m.first_row + r, load8(x + r * ldx + c, n)));
}

// ---- sums over a row ----------------------------------------------------------------
// One or two sums over the workgroup's threads, the same bits in every thread.  One barrier: the wavefronts' parts alternate between
// two places, and whoever writes a place again has passed the barrier behind the sum in between.
template <int NT>
struct RowSums {
    float* s;                                   // LDS: 2 x 2 x NT / 64
    int turn;
    __device__ __forceinline__ void operator()(float& a, float& b) {
#pragma unroll
        for (int o = 32; o; o >>= 1) {
            a += __shfl_xor(a, o);
            b += __shfl_xor(b, o);
        }
        if (NT == 64) return;
        constexpr int W = NT / 64;
        float* p = s + turn * 2 * W;
        turn ^= 1;
        if ((threadIdx.x & 63) == 0) {
            p[threadIdx.x >> 6] = a;
            p[W + (threadIdx.x >> 6)] = b;
        }
        __syncthreads();
        a = b = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            a += p[w];
            b += p[W + w];
        }
    }
    __device__ __forceinline__ void operator()(float& a) {
        float none = 0.f;
        (*this)(a, none);
    }
};
__device__ __forceinline__ float sum8(f32x8 v) { return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7])); }
// v - mean in the n columns that exist, 0 elsewhere
__device__ __forceinline__ f32x8 centred(f32x8 v, float mean, int n) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? v[i] - mean : 0.f;
    return v;
}
__device__ __forceinline__ float logistic1(float z) { return __builtin_amdgcn_rcpf(1.f + __expf(-z)); }
__device__ __forceinline__ f32x8 logistic(f32x8 z) {
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = logistic1(z[i]);
    return z;
}

template <typename T>
using raw_of = std::conditional_t<std::is_same<T, float>::value, f32x8, bf16x8>;
template <typename T>
__device__ __forceinline__ f32x8 wide(raw_of<T> v) { return __builtin_convertvector(v, f32x8); }
template <typename T>
__device__ __forceinline__ raw_of<T> raw8(const T* p, int n) {
    typedef raw_of<T> any __attribute__((aligned(sizeof(T))));
    if (n >= 8) return *(const HOPL_GLOBAL any*)p;
    raw_of<T> v = (T)0.f;
#pragma unroll
    for (int i = 0; i < 7; ++i)
        if (i < n) v[i] = ((const HOPL_GLOBAL T*)p)[i];
    return v;
}

// A workgroup takes a piece of consecutive rows of one group, so the group's vectors are read once for all of them; the next
// row's loads are on their way while a row's statistics are worked out.
template <typename T, int NT, int V>
__global__ __launch_bounds__(NT) void residual_kernel(HopResidualTask t, HopIndex index) {
    __shared__ float shared[4 * (NT / 64)];
    RowSums<NT> sums{shared, 0};
    int g, r0, r1;
    if (!find_piece(t.rows, t.shift, blockIdx.x, &g, &r0, &r1)) return;
    const int at = t.indexed ? index.at[g] : g;
    int col[V], n[V];
    f32x8 post[V], pre[V], gate[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        col[i] = (i * NT + threadIdx.x) * 8;
        n[i] = min(t.cols - col[i], 8);
        post[i] = t.post && n[i] > 0 ? load8(t.post + at * t.post_stride + col[i], n[i]) : f32x8(1.f);
        pre[i] = t.pre && n[i] > 0 ? load8(t.pre + at * t.pre_stride + col[i], n[i]) : f32x8(1.f);
        gate[i] = t.gate && n[i] > 0 ? load8(t.gate + at * t.gate_stride + col[i], n[i]) : f32x8(1.f);
    }
    raw_of<T> nx[V], nb[V], nz[V];
    auto fetch = [&](int r) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            nx[i] = nb[i] = nz[i] = (T)0.f;
            if (n[i] <= 0) continue;
            nx[i] = raw8((const T*)t.x + r * t.ldx + col[i], n[i]);
            if (t.b) nb[i] = raw8((const T*)t.b + r * t.ldb + col[i], n[i]);
            if (t.z) nz[i] = raw8((const T*)t.z + r * t.ldz + col[i], n[i]);
        }
    };
    fetch(r0);
    for (int r = r0; r < r1; ++r) {
        f32x8 x[V], b[V], z[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            x[i] = wide<T>(nx[i]);
            b[i] = wide<T>(nb[i]);
            z[i] = wide<T>(nz[i]);
        }
        if (r + 1 < r1) fetch(r + 1);
        if (t.b) {
            if (t.norm == HOP_NORM_CENTRED) {
                float a = 0.f;
#pragma unroll
                for (int i = 0; i < V; ++i) a += sum8(b[i]);
                sums(a);
#pragma unroll
                for (int i = 0; i < V; ++i) b[i] = centred(b[i], a * t.inv_cols, n[i]);
            }
            if (t.norm) {
                float a = 0.f;
#pragma unroll
                for (int i = 0; i < V; ++i) a += sum8(b[i] * b[i]);
                sums(a);
                a = rsqrtf(a * t.inv_cols + t.eps);
#pragma unroll
                for (int i = 0; i < V; ++i) b[i] *= a;
            }
#pragma unroll
            for (int i = 0; i < V; ++i) {
                f32x8 u = b[i] * post[i] * gate[i];
                if (t.z) u *= logistic(z[i]);
                if (t.mask.threshold) u = dropped(t.mask, col[i] >> 3, t.mask.first_row + r, u);
                x[i] += t.scale * u;
                if (n[i] > 0) store8((T*)t.y + r * t.ldy + col[i], n[i], x[i]);
            }
        }
        if (t.h) {
            if (t.next_norm == HOP_NORM_CENTRED) {
                float a = 0.f;
#pragma unroll
                for (int i = 0; i < V; ++i) a += sum8(x[i]);       // columns that do not exist hold 0
                sums(a);
#pragma unroll
                for (int i = 0; i < V; ++i) x[i] = centred(x[i], a * t.inv_cols, n[i]);
            }
            float a = 0.f;
#pragma unroll
            for (int i = 0; i < V; ++i) a += sum8(x[i] * x[i]);
            sums(a);
            a = rsqrtf(a * t.inv_cols + t.eps);
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (n[i] > 0) store8((T*)t.h + r * t.ldh + col[i], n[i], x[i] * a * pre[i]);
        }
    }
}

// n = norm(v) in place; r: its factor
template <int NT, int V>
__device__ __forceinline__ void normalise(f32x8 (&v)[V], const int (&n)[V], int norm, float inv_cols, float eps, float* r, RowSums<NT>& sums) {
    if (norm == HOP_NORM_CENTRED) {
        float a = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) a += sum8(v[i]);
        sums(a);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = centred(v[i], a * inv_cols, n[i]);
    }
    float a = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) a += sum8(v[i] * v[i]);
    sums(a);
    *r = rsqrtf(a * inv_cols + eps);
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] *= *r;
}
// a <- r (a - [mean a] - n mean(a n)): the gradient through a norm whose result was n; 0 in columns that do not exist
template <int NT, int V>
__device__ __forceinline__ void through_norm(f32x8 (&a)[V], const f32x8 (&nv)[V], const int (&n)[V], int norm, float inv_cols, float r, RowSums<NT>& sums) {
    float s = 0.f, sn = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        s += sum8(a[i]);
        sn += sum8(a[i] * nv[i]);
    }
    sums(s, sn);
    sn *= inv_cols;
    if (norm == HOP_NORM_CENTRED) {
#pragma unroll
        for (int i = 0; i < V; ++i) a[i] = centred(a[i], s * inv_cols, n[i]);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) a[i] = r * (a[i] - nv[i] * sn);
}

template <typename T, int NT, int V>
__global__ __launch_bounds__(NT) void residual_grad_kernel(HopResidualTask t, HopIndex index) {
    __shared__ float shared[4 * (NT / 64)];
    RowSums<NT> sums{shared, 0};
    int g, r0, r1;
    if (!find_piece(t.rows, t.shift, blockIdx.x, &g, &r0, &r1)) return;
    const int at = t.indexed ? index.at[g] : g;
    int col[V], n[V];
    f32x8 dpost[V] = {}, dpre[V] = {}, dgate[V] = {};
#pragma unroll
    for (int i = 0; i < V; ++i) {
        col[i] = (i * NT + threadIdx.x) * 8;
        n[i] = min(t.cols - col[i], 8);
    }
    auto vector = [&](const float* p, int64_t stride, int i) {
        return p && n[i] > 0 ? load8(p + at * stride + col[i], n[i]) : f32x8(1.f);
    };
    auto matrix = [&](const void* p, int64_t ld, int r, int i) {
        return p && n[i] > 0 ? wide<T>(raw8((const T*)p + r * ld + col[i], n[i])) : f32x8(0.f);
    };
    for (int r = r0; r < r1; ++r) {
        f32x8 e[V], a[V], v[V], b[V], z[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            e[i] = matrix(t.dy, t.lddy, r, i);
            a[i] = matrix(t.dh, t.lddh, r, i);
            v[i] = t.dh ? matrix(t.y, t.ldy, r, i) : f32x8(0.f);
            b[i] = matrix(t.b, t.ldb, r, i);
            z[i] = matrix(t.z, t.ldz, r, i);
        }
        if (t.dh) {
            float f;
            normalise<NT, V>(v, n, t.next_norm, t.inv_cols, t.eps, &f, sums);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                dpre[i] += a[i] * v[i];
                a[i] *= vector(t.pre, t.pre_stride, i);
            }
            through_norm<NT, V>(a, v, n, t.next_norm, t.inv_cols, f, sums);
#pragma unroll
            for (int i = 0; i < V; ++i) e[i] += a[i];
        }
        if (t.dx) {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (n[i] > 0) store8((T*)t.dx + r * t.lddx + col[i], n[i], e[i]);
        }
        if (!t.b) continue;
        float rb = 1.f;
        if (t.norm) normalise<NT, V>(b, n, t.norm, t.inv_cols, t.eps, &rb, sums);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            f32x8 f = e[i];
            if (t.mask.threshold) f = dropped(t.mask, col[i] >> 3, t.mask.first_row + r, f);
            f *= t.scale;
            const f32x8 post = vector(t.post, t.post_stride, i);
            if (t.z) {
                const f32x8 s = logistic(z[i]);
                if (t.dz && n[i] > 0) store8((T*)t.dz + r * t.lddz + col[i], n[i], f * b[i] * post * s * (1.f - s));
                f *= s;
            } else if (t.gate) {
                dgate[i] += f * b[i] * post;
                f *= vector(t.gate, t.gate_stride, i);
            }
            dpost[i] += f * b[i];
            a[i] = f * post;
        }
        if (t.db) {
            if (t.norm) through_norm<NT, V>(a, b, n, t.norm, t.inv_cols, rb, sums);
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (n[i] > 0) store8((T*)t.db + r * t.lddb + col[i], n[i], a[i]);
        }
    }
    if (!t.partial) return;
    float* p = t.partial + (int64_t)blockIdx.x * 3 * t.cols;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if (n[i] <= 0) continue;
        if (t.dpost) store8(p + col[i], n[i], dpost[i]);
        if (t.dpre) store8(p + t.cols + col[i], n[i], dpre[i]);
        if (t.dgate) store8(p + 2 * (int64_t)t.cols + col[i], n[i], dgate[i]);
    }
}

// The pieces of group g: the first and how many, as find_piece numbers them.
__device__ __forceinline__ void group_pieces(const HopRows& rows, int shift, int g, int* first, int* count) {
    const int step = 1 << shift;
    if (!rows.begin) {
        *first = 0;
        *count = (int)(((int64_t)rows.rows + step - 1) >> shift);
        return;
    }
    const int lane = threadIdx.x & 63;
    const HOPL_GLOBAL int32_t* table = (const HOPL_GLOBAL int32_t*)rows.begin;
    int before = 0, mine = 0;
    for (int at = lane; at <= g; at += 64) {
        const int b = clamp_int(table[at], 0, rows.rows), e = clamp_int(table[at + 1], b, rows.rows);
        const int pieces = (int)(((int64_t)(e - b) + step - 1) >> shift);
        if (at < g) before += pieces;
        else mine = pieces;
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) {
        before += __shfl_xor(before, o);
        mine += __shfl_xor(mine, o);
    }
    *first = before;
    *count = mine;
}

// Gradients of parameters: the pieces' sums of a group, joined in a fixed order.
template <int WAVES>
__global__ __launch_bounds__(WAVES * 64) void residual_join_kernel(HopResidualTask t, int chunks, HopIndex dindex) {
    __shared__ float s[WAVES][64];
    const int g = blockIdx.y, which = blockIdx.z, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float* out = which == 0 ? t.dpost : which == 1 ? t.dpre : t.dgate;
    if (!out) return;
    out += (t.dindexed ? dindex.at[g] : g) * (which == 0 ? t.dpost_stride : which == 1 ? t.dpre_stride : t.dgate_stride);
    int first, count;
    group_pieces(t.rows, t.shift, g, &first, &count);
    first = clamp_int(first, 0, chunks);
    count = clamp_int(count, 0, chunks - first);
    const int col = blockIdx.x * 64 + lane;
    float a = 0.f;
    if (col < t.cols) {
        const float* p = t.partial + ((int64_t)first * 3 + which) * t.cols + col;
#pragma unroll 8
        for (int c = wave; c < count; c += WAVES) a += p[(int64_t)c * 3 * t.cols];
    }
    s[wave][lane] = a;
    __syncthreads();
    if (wave || col >= t.cols) return;
    a = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) a += s[w][lane];
    out[col] = a;
}

constexpr int64_t kMostPieces = 1 << 18;        // times 1024 threads: well below what a grid can have

int64_t pieces_of(int64_t rows, int G, int shift) { return (rows >> shift) + (G < rows ? G : rows); }

template <typename T, int NT, int V>
void launch(const HopResidualTask& t, const HopIndex& index, int64_t pieces, bool grad, hipStream_t st) {
    if (grad) residual_grad_kernel<T, NT, V><<<dim3((unsigned)pieces), NT, 0, st>>>(t, index);
    else residual_kernel<T, NT, V><<<dim3((unsigned)pieces), NT, 0, st>>>(t, index);
}
template <typename T>
void launch(const HopResidualTask& t, const HopIndex& index, int64_t pieces, bool grad, hipStream_t st) {
    if (t.cols <= 512) launch<T, 64, 1>(t, index, pieces, grad, st);
    else if (t.cols <= 1024) launch<T, 128, 1>(t, index, pieces, grad, st);
    else if (t.cols <= 2048) launch<T, 256, 1>(t, index, pieces, grad, st);
    else if (t.cols <= 4096) launch<T, 512, 1>(t, index, pieces, grad, st);
    else if (t.cols <= 8192) launch<T, 1024, 1>(t, index, pieces, grad, st);
    else if (t.cols <= 16384) launch<T, 1024, 2>(t, index, pieces, grad, st);
    else launch<T, 1024, 4>(t, index, pieces, grad, st);
}

}  // namespace

int hopl_dropout(int dtype, const void* x, int64_t ldx, void* y, int64_t ldy, int64_t rows, int64_t cols, const HopMask& m, void* stream) {
    hipStream_t st = (hipStream_t)stream;
    const dim3 grid((unsigned)((cols + 2047) / 2048), (unsigned)(rows < 65535 ? rows : 65535));
    if (dtype == HOP_BF16) dropout_kernel<bf16><<<grid, 256, 0, st>>>((const bf16*)x, ldx, (bf16*)y, ldy, rows, cols, m);
    else dropout_kernel<float><<<grid, 256, 0, st>>>((const float*)x, ldx, (float*)y, ldy, rows, cols, m);
    return (int)hipGetLastError();
}

int hopl_residual(HopResidualTask t, int dtype, const HopIndex& index, void* stream) {
    t.shift = 0;
    while ((t.shift < 5 && (t.rows.rows >> (t.shift + 1)) >= 4096) || (t.rows.rows >> t.shift) > kMostPieces) ++t.shift;
    const int64_t pieces = pieces_of(t.rows.rows, t.rows.G, t.shift);
    if (dtype == HOP_BF16) launch<bf16>(t, index, pieces, false, (hipStream_t)stream);
    else launch<float>(t, index, pieces, false, (hipStream_t)stream);
    return (int)hipGetLastError();
}

int hopl_grad_shift(int64_t rows, int G, int64_t cols) {
    (void)G, (void)cols;
    int shift = 0;
    while ((shift < 7 && (rows >> (shift + 1)) >= 768) || (rows >> shift) > kMostPieces) ++shift;
    return shift;
}
int64_t hopl_grad_chunks(int64_t rows, int G, int64_t cols) { return pieces_of(rows, G, hopl_grad_shift(rows, G, cols)); }

int hopl_residual_grad(HopResidualTask t, int dtype, const HopIndex& index, const HopIndex& dindex, void* stream) {
    hipStream_t st = (hipStream_t)stream;
    t.shift = hopl_grad_shift(t.rows.rows, t.rows.G, t.cols);
    const int64_t chunks = pieces_of(t.rows.rows, t.rows.G, t.shift);
    if (chunks > 0) {
        if (dtype == HOP_BF16) launch<bf16>(t, index, chunks, true, st);
        else launch<float>(t, index, chunks, true, st);
    }
    if (t.dpost || t.dpre || t.dgate) {
        const dim3 grid((unsigned)((t.cols + 63) / 64), (unsigned)t.rows.G, 3);
        if (chunks / t.rows.G > 32) residual_join_kernel<16><<<grid, 1024, 0, st>>>(t, (int)chunks, dindex);
        else residual_join_kernel<4><<<grid, 256, 0, st>>>(t, (int)chunks, dindex);
    }
    return (int)hipGetLastError();
}
