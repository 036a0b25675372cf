// Norm and rotation of the heads of queries and keys in one pass, and its gradients, for gfx950 (CDNA4).
//
//   n = norm(x_h),  t = n w,  y = R(position) t;  u = R(-position) dy,  dw = sum u n,  dx = norm'(u w; x)
//
// A few dozen operations an element: what bounds it is reading x (and dy) and writing y (dx) once, 16384 rows of 40 heads of 128 columns in bfloat16 in 74 us (4.5 TB/s), gradients
// in 117 (4.3; a copy of as much reaches 5.3).  A head belongs to a few neighbouring lanes, eight columns
// each, so its statistics and the other column of a pair are a few exchanges between lanes away; the sines and cosines of four rows at a time are worked
// out by one lane each and shared by all their heads.
#include <algorithm>

#include "hop_attention_internal.h"
#include "hop_layers_device.h"

using namespace hopl;

namespace {

constexpr int NT = 256, kBlock = 4, kMostPairs = HOP_MAX_HEAD_COLS / 2;       // rows whose angles are worked out at once
// Where the other column of a pair is: in the lane half a head away (halves of whole heads of 2^k columns), in the same lane (neighbours), or anywhere in the head.
enum { kLanes, kNeighbours, kAnywhere };

struct Shared {
    float cosine[kBlock][kMostPairs], sine[kBlock][kMostPairs];
    float exchange[NT * 8];
};

__device__ __forceinline__ int position_of(const HopRotateTask& t, int row) {
    if (t.positions) return ((const HOPL_GLOBAL int32_t*)t.positions)[row];
    if (!t.sequences.begin) return row;
    const HOPL_GLOBAL int32_t* table = (const HOPL_GLOBAL int32_t*)t.sequences.begin;
    const int lane = threadIdx.x & 63;
    int from = 0;
    for (int base = 0; base < t.sequences.G; base += 64) {                    // the last sequence that begins at or in front of the row
        const int b = base + lane < t.sequences.G ? table[base + lane] : 0x7FFFFFFF;
        const uint64_t before = __ballot(b <= row);
        if (before) from = __builtin_amdgcn_readlane(b, 63 - __builtin_clzll(before));
        if (before != ~0ull) break;
    }
    return row - from;
}

// Angles of up to kBlock rows from r0 on: a wavefront a row, a lane a pair.  The product of position and frequency is held in 64 bits, in
// turns, of which the nearest whole number is taken off; what is left, at most half a turn, is rounded to 32.
__device__ __forceinline__ void angles(const HopRotateTask& t, Shared& sh, int r0, int rows) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    if (wave < rows && t.rotary) {
        const int position = position_of(t, r0 + wave);
        if (lane < t.rotary / 2) {
            double turns = (double)position * t.turns[lane];
            turns -= __builtin_rint(turns);
            float s, c;
            sincospif((float)(2.0 * turns), &s, &c);
            sh.cosine[wave][lane] = c;
            sh.sine[wave][lane] = s;
        }
    }
    __syncthreads();
}

// A value of another lane of the same 16, without LDS: quad_perm 0 to 0xFF, row_shl 0x100 + n, row_shr 0x110 + n, row_ror 0x120 + n, row_mirror 0x140, row_half_mirror 0x141.
template <int CONTROL, int BANKS = 15>
__device__ __forceinline__ float moved(float old, float v) {
    return __uint_as_float(__builtin_amdgcn_update_dpp(__float_as_uint(old), __float_as_uint(v), CONTROL, 15, BANKS, false));
}
// The sum over the lanes of a head, 1, 2, 4, 8 or 16 of them; what a step adds is the same in all lanes of the other half, so a mirror will do.
__device__ __forceinline__ float head_sum(float v, int lanes) {
    if (lanes > 1) v += moved<0xB1>(v, v);
    if (lanes > 2) v += moved<0x4E>(v, v);
    if (lanes > 4) v += moved<0x141>(v, v);
    if (lanes > 8) v += moved<0x140>(v, v);
    return v;
}
// The columns of the lane half a head away.
__device__ __forceinline__ f32x8 half_away(f32x8 v, int lanes) {
    f32x8 r;
    if (lanes == 16) {
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = moved<0x128>(v[e], v[e]);
    } else if (lanes == 8) {
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = moved<0x114, 10>(moved<0x104, 5>(v[e], v[e]), v[e]);
    } else if (lanes == 4) {
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = moved<0x4E>(v[e], v[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = moved<0xB1>(v[e], v[e]);
    }
    return r;
}

// The columns from c0 on turned by the angles of row `r` of the block; `back`: by their negatives.
template <int MODE>
__device__ __forceinline__ f32x8 turn(const HopRotateTask& t, Shared& sh, f32x8 v, int r, int c0, int lanes, bool back) {
    f32x8 other, cosine, sine;
    const int half = t.rotary / 2;
    if constexpr (MODE == kLanes) {
        const int i = c0 & (half - 1);
        const float sign = (c0 < half) != back ? -1.f : 1.f;
        cosine = *(const f32x8*)&sh.cosine[r][i];
        sine = *(const f32x8*)&sh.sine[r][i];
        other = half_away(v, lanes);
        sine *= sign;
    } else if constexpr (MODE == kNeighbours) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int c = c0 + e, i = c / 2 < half ? c / 2 : 0;
            const bool turned = c < t.rotary;
            other[e] = v[e ^ 1];
            cosine[e] = turned ? sh.cosine[r][i] : 1.f;
            sine[e] = turned ? ((e & 1) == 0) != back ? -sh.sine[r][i] : sh.sine[r][i] : 0.f;
        }
    } else {
        float* mine = sh.exchange + (threadIdx.x & ~(lanes - 1)) * 8;
        __builtin_amdgcn_wave_barrier();
        *(f32x8*)(mine + c0) = v;
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int c = c0 + e;
            const bool turned = c < t.rotary, first = c < half;
            const int i = !turned ? 0 : first ? c : c - half, at = !turned ? c : first ? c + half : c - half;
            other[e] = mine[at];
            cosine[e] = turned ? sh.cosine[r][i] : 1.f;
            sine[e] = turned ? first != back ? -sh.sine[r][i] : sh.sine[r][i] : 0.f;
        }
    }
    f32x8 y;
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = __builtin_fmaf(other[e], sine[e], v[e] * cosine[e]);
    return y;
}

__device__ __forceinline__ float sum8(f32x8 v) { return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7])); }

// n = norm(x) of the lane's columns, `exist` of them; returns the factor of the norm.
__device__ __forceinline__ float normed(const HopRotateTask& t, f32x8& x, int exist, int lanes) {
    if (t.norm == HOP_NORM_NONE) return 1.f;
    if (t.norm == HOP_NORM_CENTRED) {
        const float mean = head_sum(sum8(x), lanes) * t.inv_cols;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = e < exist ? x[e] - mean : 0.f;
    }
    float squares = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) squares = __builtin_fmaf(x[e], x[e], squares);
    const float r = 1.f / __builtin_sqrtf(__builtin_fmaf(head_sum(squares, lanes), t.inv_cols, t.eps));
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= r;
    return r;
}

// A lane's eight columns of a parameter; ones where there is none.
__device__ __forceinline__ f32x8 weights(const float* w, int64_t stride, int at, int c0, int exist) {
    if (!w || exist <= 0) return (f32x8)(1.f);
    return load8(w + at * stride + c0, exist);
}

// Eight columns as they lie in memory, zeros where there is none.
// How many of a thread's heads are on their way at once.  16384 rows of 40 heads of 128 columns in bfloat16: two 73 us, one 77; fp32, 8192 rows of 16 heads of 64: 19, one 17.
template <typename T>
constexpr int kHeads = sizeof(T) == 2 ? 2 : 1;
template <typename T>
struct Columns;
template <>
struct Columns<bf16> {
    typedef bf16x8 type;
    static __device__ __forceinline__ type load(const bf16* p, int exist) {
        if (exist >= 8) return *(const HOPL_GLOBAL bf16x8_any*)p;
        if (exist <= 0) return (bf16x8)((bf16)0.f);
        return load_short<bf16x8>(p, exist);
    }
    static __device__ __forceinline__ f32x8 wide(type v) { return __builtin_convertvector(v, f32x8); }
};
template <>
struct Columns<float> {
    typedef f32x8 type;
    static __device__ __forceinline__ type load(const float* p, int exist) { return exist <= 0 ? (f32x8)(0.f) : load8(p, exist); }
    static __device__ __forceinline__ f32x8 wide(type v) { return v; }
};

template <typename T, int MODE>
__global__ __launch_bounds__(NT) void rotate_kernel(HopRotateTask t, HopIndex index, int lanes) {
    __shared__ __attribute__((aligned(32))) Shared sh;
    int g, r0, r1;
    if (!find_piece(t.rows, t.shift, blockIdx.x, &g, &r0, &r1)) return;
    const int at = t.indexed ? index.at[g] : g;
    const int slots = NT / lanes, slot = threadIdx.x / lanes, c0 = (threadIdx.x & (lanes - 1)) * 8, exist = t.cols - c0;
    const f32x8 wq = weights(t.q_weight, t.q_stride, at, c0, exist), wk = weights(t.k_weight, t.k_stride, at, c0, exist);
    for (int from = r0; from < r1; from += kBlock) {
        const int rows = min(kBlock, r1 - from);
        int r = 0, h = slot;
        auto settle = [&] {
            while (h >= t.heads) {
                h -= t.heads;
                ++r;
            }
        };
        settle();
        const T* x = (const T*)t.x + from * t.ldx + c0;
        T* y = (T*)t.y + from * t.ldy + c0;
        // Heads on their way: kHeads<T> at once, the first ones while the angles are worked out.
        typename Columns<T>::type v[kHeads<T>];
        int rs[kHeads<T>], hs[kHeads<T>];
        auto fetch = [&](int i) __attribute__((always_inline)) {
            rs[i] = r;
            hs[i] = h;
            if (r < rows) v[i] = Columns<T>::load(x + r * t.ldx + h * t.cols, exist);
            h += slots;
            settle();
        };
#pragma unroll
        for (int i = 0; i < kHeads<T>; ++i) fetch(i);
        if (from > r0) __syncthreads();
        angles(t, sh, from, rows);
        while (rs[0] < rows) {
#pragma unroll
            for (int i = 0; i < kHeads<T>; ++i) {
                const int this_r = rs[i], this_h = hs[i];
                if (this_r >= rows) break;
                f32x8 n = Columns<T>::wide(v[i]);
                fetch(i);
                normed(t, n, exist, lanes);
                n *= this_h < t.q_heads ? wq : wk;
                n = turn<MODE>(t, sh, n, this_r, c0, lanes, false);
                if (exist > 0) store8(y + this_r * t.ldy + this_h * t.cols, exist, n);
            }
        }
    }
}

// Four wavefronts to a SIMD are all of 1024 workgroups at once: 117 us for 16384 rows of 40 heads of 128 columns in bfloat16; a register more than that allows, 169.
template <typename T, int MODE>
__global__ __launch_bounds__(NT, 4) void rotate_grad_kernel(HopRotateTask t, HopIndex index, int lanes) {
    __shared__ __attribute__((aligned(32))) Shared sh;
    int g, r0, r1;
    if (!find_piece(t.rows, t.shift, blockIdx.x, &g, &r0, &r1)) return;
    const int at = t.indexed ? index.at[g] : g;
    const int slots = NT / lanes, slot = threadIdx.x / lanes, c0 = (threadIdx.x & (lanes - 1)) * 8, exist = t.cols - c0;
    const f32x8 wq = weights(t.q_weight, t.q_stride, at, c0, exist), wk = weights(t.k_weight, t.k_stride, at, c0, exist);
    f32x8 dq = (f32x8)(0.f), dk = (f32x8)(0.f);
    for (int from = r0; from < r1; from += kBlock) {
        const int rows = min(kBlock, r1 - from);
        int r = 0, h = slot;
        auto settle = [&] {
            while (h >= t.heads) {
                h -= t.heads;
                ++r;
            }
        };
        settle();
        const T *x = (const T*)t.x + from * t.ldx + c0, *dy = (const T*)t.dy + from * t.lddy + c0;
        T* dx = (T*)t.dx + from * t.lddx + c0;
        f32x8 vx = (f32x8)(0.f), vy = (f32x8)(0.f);
        auto fetch = [&] {
            if (r >= rows) return;
            vx = Columns<T>::wide(Columns<T>::load(x + r * t.ldx + h * t.cols, exist));
            vy = Columns<T>::wide(Columns<T>::load(dy + r * t.lddy + h * t.cols, exist));
        };
        fetch();                                                                    // on its way while the angles are worked out
        if (from > r0) __syncthreads();
        angles(t, sh, from, rows);
        while (r < rows) {
            const int this_r = r, this_h = h;
            f32x8 n = vx, u = vy;
            h += slots;
            settle();
            fetch();
            const float factor = normed(t, n, exist, lanes);
            u = turn<MODE>(t, sh, u, this_r, c0, lanes, true);
            if (this_h < t.q_heads) {
                dq += u * n;
                u *= wq;
            } else {
                dk += u * n;
                u *= wk;
            }
            if (!t.dx) continue;
            if (t.norm != HOP_NORM_NONE) {
                const float along = head_sum(sum8(u * n), lanes) * t.inv_cols;
                const float mean = t.norm == HOP_NORM_CENTRED ? head_sum(sum8(u), lanes) * t.inv_cols : 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) u[e] = (u[e] - n[e] * along - mean) * factor;
            }
            if (exist > 0) store8(dx + this_r * t.lddx + this_h * t.cols, exist, u);
        }
    }
    if (!t.partial) return;
    // the slots' sums, in their order
    for (int which = 0; which < 2; ++which) {
        __syncthreads();
        *(f32x8*)(sh.exchange + threadIdx.x * 8) = which ? dk : dq;
        __syncthreads();
        for (int c = threadIdx.x; c < t.cols; c += NT) {
            float sum = 0.f;
            for (int i = 0; i < slots; ++i) sum += sh.exchange[i * lanes * 8 + c];
            ((HOPL_GLOBAL float*)t.partial)[((int64_t)blockIdx.x * 2 + which) * t.cols + c] = sum;
        }
    }
}

// The chunks of a group, summed: 16 columns a workgroup, 64 threads a column, each an even share of the chunks in their order.
constexpr int kShares = 64;
__global__ __launch_bounds__(16 * kShares) void rotate_join_kernel(HopRotateTask t, HopIndex index) {
    __shared__ float sums[kShares][17];
    const int g = blockIdx.x, which = blockIdx.y, column = threadIdx.x & 15, share = threadIdx.x >> 4, c = blockIdx.z * 16 + column;
    float* to = which ? t.dk_weight : t.dq_weight;
    if (!to) return;
    HopRows before = t.rows;
    before.G = g;
    const int first = t.rows.begin ? count_pieces(before, t.shift) : 0;
    int b, e;
    group_rows(t.rows, g, &b, &e);
    const int pieces = (int)(((int64_t)(e - b) + (1 << t.shift) - 1) >> t.shift), each = (pieces + kShares - 1) / kShares;
    const HOPL_GLOBAL float* from = (const HOPL_GLOBAL float*)t.partial + ((int64_t)first * 2 + which) * t.cols + c;
    float sum = 0.f;
    if (c < t.cols)
#pragma unroll 8
        for (int i = share * each; i < min(pieces, (share + 1) * each); ++i) sum += from[(int64_t)i * 2 * t.cols];
    sums[share][column] = sum;
    __syncthreads();
    if (share || c >= t.cols) return;
    for (int i = 1; i < kShares; ++i) sum += sums[i][column];
    ((HOPL_GLOBAL float*)to)[(t.dindexed ? index.at[g] : g) * (which ? t.dk_stride : t.dq_stride) + c] = sum;
}

int lanes_of(int cols) {
    int n = 1;
    while (n * 8 < cols) n *= 2;
    return n;
}
int mode_of(const HopRotateTask& t) {
    if (t.adjacent) return kNeighbours;
    const int lanes = lanes_of(t.cols);
    return t.rotary == t.cols && lanes * 8 == t.cols && lanes > 1 ? kLanes : kAnywhere;
}

template <typename T>
void forward(const HopRotateTask& t, const HopIndex& index, unsigned grid, hipStream_t stream) {
    const int lanes = lanes_of(t.cols);
    switch (mode_of(t)) {
        case kLanes: rotate_kernel<T, kLanes><<<dim3(grid), dim3(NT), 0, stream>>>(t, index, lanes); break;
        case kNeighbours: rotate_kernel<T, kNeighbours><<<dim3(grid), dim3(NT), 0, stream>>>(t, index, lanes); break;
        default: rotate_kernel<T, kAnywhere><<<dim3(grid), dim3(NT), 0, stream>>>(t, index, lanes);
    }
}
template <typename T>
void backward(const HopRotateTask& t, const HopIndex& index, unsigned grid, hipStream_t stream) {
    const int lanes = lanes_of(t.cols);
    switch (mode_of(t)) {
        case kLanes: rotate_grad_kernel<T, kLanes><<<dim3(grid), dim3(NT), 0, stream>>>(t, index, lanes); break;
        case kNeighbours: rotate_grad_kernel<T, kNeighbours><<<dim3(grid), dim3(NT), 0, stream>>>(t, index, lanes); break;
        default: rotate_grad_kernel<T, kAnywhere><<<dim3(grid), dim3(NT), 0, stream>>>(t, index, lanes);
    }
}

}  // namespace

int hopa_rotate(const HopRotateTask& task, int dtype, const HopIndex& index, void* stream) {
    HopRotateTask t = task;
    t.shift = t.rows.rows > 2048 ? 2 : 0;
    while ((t.rows.rows >> t.shift) > kHopaMostChunks) ++t.shift;
    const unsigned grid = (unsigned)(((int64_t)t.rows.rows + (1 << t.shift) - 1) / (1 << t.shift) + (t.rows.begin ? t.rows.G : 0));
    if (dtype == HOP_BF16) forward<bf16>(t, index, grid, (hipStream_t)stream);
    else forward<float>(t, index, grid, (hipStream_t)stream);
    return (int)hipGetLastError();
}

int hopa_rotate_grad(const HopRotateTask& task, int dtype, const HopIndex& index, const HopIndex& dindex, void* stream) {
    HopRotateTask t = task;
    t.shift = hopa_rotate_shift(t.rows.rows);
    if (t.rows.rows) {
        const unsigned grid = (unsigned)hopa_rotate_chunks(t.rows.rows, t.rows.begin ? t.rows.G : 0);
        if (dtype == HOP_BF16) backward<bf16>(t, index, grid, (hipStream_t)stream);
        else backward<float>(t, index, grid, (hipStream_t)stream);
    }
    if (t.dq_weight || t.dk_weight)
        rotate_join_kernel<<<dim3((unsigned)t.rows.G, 2, (unsigned)((t.cols + 15) / 16)), dim3(16 * kShares), 0, (hipStream_t)stream>>>(t, dindex);
    return (int)hipGetLastError();
}
