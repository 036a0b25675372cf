// Norms before and after a block fused with its gate, dropout and residual sum, their gradients, and dropout by itself, for gfx950.
//
//   n = norm(b), t = n post, u = gate t, y = x + scale dropout(u), h = next_norm(y) pre
//   e = dy + next_norm'(dh pre; y), f = scale dropout(e), q = f gate, db = norm'(q post; b), norm'(a; v) = r (a - [mean a] - n mean(a n))
//
// A row is read once, stays in registers through its statistics (eight consecutive columns a thread), and is written once; the mask is worked
// out again wherever it is needed.  That holds up to 8192 columns: wider rows' kernels spill 50 to 200 registers a thread, over 16384 up to 1700.  The next
// row is loaded ahead where rows are whole pieces of eight columns; elsewhere the loads wait for each other (see columns8).  About 39 vector instructions an element forwards and 54 back, the generator's among them, so instruction issue comes
// close behind the bytes: 16384 x 4096 in bf16 with dropout 103 us forwards (5.2 TB/s of the 537 MB), 170 back (4.7 TB/s of 805); dropout of
// 8192 x 8192 in bf16 48 us (5.6 TB/s).  With few rows the chain of a row - loads, two to four sums over the workgroup - bounds it: 8 rows of 4096 5.6 us.
#include <type_traits>

#include "hop_layers_device.h"

using namespace hopl;

namespace {

template <typename T>
using raw_of = std::conditional_t<std::is_same<T, float>::value, f32x8, bf16x8>;
template <typename T>
__device__ __forceinline__ f32x8 wide(raw_of<T> v) { return __builtin_convertvector(v, f32x8); }
// Eight columns of a row from byte `at` on, as they are; n <= 8 of them exist (n <= 0: none), the rest are zero.  At the end of a row that is no
// multiple of eight, the row's last eight are loaded and moved down: single loads there held a register pair each, or waited
// for each other.  `at` is 32 bits wide and `line` the same for all threads, so an address takes one register.  Whether to move down is a
// branch on what was loaded, so a load's wait stands right behind it.
__device__ __forceinline__ u32x4 moved_down(u32x4 v, int by) {          // by elements of 16 bits
    if (by & 4) v = u32x4{v[2], v[3], 0, 0};
    if (by & 2) v = u32x4{v[1], v[2], v[3], 0};
    if (by & 1) v = u32x4{v[0] >> 16 | v[1] << 16, v[1] >> 16 | v[2] << 16, v[2] >> 16 | v[3] << 16, v[3] >> 16};
    return v;
}
__device__ __forceinline__ f32x8 moved_down(f32x8 v, int by) {
    if (by & 4) v = f32x8{v[4], v[5], v[6], v[7], 0, 0, 0, 0};
    if (by & 2) v = f32x8{v[2], v[3], v[4], v[5], v[6], v[7], 0, 0};
    if (by & 1) v = f32x8{v[1], v[2], v[3], v[4], v[5], v[6], v[7], 0};
    return v;
}
template <typename T>
__device__ __forceinline__ raw_of<T> columns8(const T* line, int cols, uint32_t at, int n) {
    typedef raw_of<T> any __attribute__((aligned(sizeof(T))));
    typedef std::conditional_t<std::is_same<T, float>::value, f32x8, u32x4> words;
    if (n <= 0) return raw_of<T>((T)0.f);
    if (cols < 8) return load_short<raw_of<T>>(line, n);
    const uint32_t from = n >= 8 ? at : (uint32_t)(cols - 8) * (uint32_t)sizeof(T);
    raw_of<T> v = *(const HOPL_GLOBAL any*)((const HOPL_GLOBAL char*)line + from);
    if (n < 8) v = __builtin_bit_cast(raw_of<T>, moved_down(__builtin_bit_cast(words, v), 8 - n));
    return v;
}

template <typename T>
__device__ __forceinline__ void put8(T* line, uint32_t at, int n, f32x8 v) {
    typedef raw_of<T> any __attribute__((aligned(sizeof(T))));
    HOPL_GLOBAL char* p = (HOPL_GLOBAL char*)line + at;
    const raw_of<T> r = __builtin_convertvector(v, raw_of<T>);      // to nearest, ties to even
    if (n >= 8) {
        *(HOPL_GLOBAL any*)p = r;
        return;
    }
#pragma unroll
    for (int i = 0; i < 7; ++i)
        if (i < n) ((HOPL_GLOBAL T*)p)[i] = r[i];
}

// A matrix's rows, or nothing (p null: reads are zero, writes go nowhere).  EVEN: rows are whole pieces of eight columns at addresses that are
// multiples of four, and go through buffer descriptors of a row: what lies behind a row's end is then zero, or dropped, by the descriptor's
// end instead of by branches, and addresses cost no vector instructions (these kernels are bound by instruction issue as much as by bytes).
template <typename T, bool EVEN>
struct Matrix {
    T* p;
    int64_t ld;
    int cols;
    uint32_t bytes;
    __device__ __forceinline__ Matrix(const void* p_, int64_t ld_, int cols_) : p((T*)p_), ld(ld_), cols(cols_), bytes(p_ ? cols_ * (uint32_t)sizeof(T) : 0u) {}
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t row(int r) const { return __builtin_amdgcn_make_buffer_rsrc(p + r * ld, 0, (int)bytes, 0x00020000); }
    __device__ __forceinline__ raw_of<T> load(int r, uint32_t col, int n) const {
        if constexpr (EVEN) {
            const __amdgpu_buffer_rsrc_t d = row(r);
            const uint32_t at = col * (uint32_t)sizeof(T);
            const u32x4 a = __builtin_amdgcn_raw_buffer_load_b128(d, at, 0, 0);
            if constexpr (sizeof(T) == 2) return __builtin_bit_cast(raw_of<T>, a);
            else {
                const u32x4 b = __builtin_amdgcn_raw_buffer_load_b128(d, at + 16, 0, 0);
                const f32x4 u = __builtin_bit_cast(f32x4, a), v = __builtin_bit_cast(f32x4, b);
                return raw_of<T>{u[0], u[1], u[2], u[3], v[0], v[1], v[2], v[3]};
            }
        } else {
            return p ? columns8(p + r * ld, cols, col * (uint32_t)sizeof(T), n) : raw_of<T>((T)0.f);
        }
    }
    __device__ __forceinline__ void store(int r, uint32_t col, int n, f32x8 v) const {
        if constexpr (EVEN) {
            const __amdgpu_buffer_rsrc_t d = row(r);
            const uint32_t at = col * (uint32_t)sizeof(T);
            if constexpr (sizeof(T) == 2) {
                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, __builtin_convertvector(v, bf16x8)), d, at, 0, 0);
            } else {
                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f32x4{v[0], v[1], v[2], v[3]}), d, at, 0, 0);
                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f32x4{v[4], v[5], v[6], v[7]}), d, at + 16, 0, 0);
            }
        } else if (p && n > 0) {
            put8(p + r * ld, col * (uint32_t)sizeof(T), n, v);
        }
    }
};

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
// Which of eight columns the mask keeps.  A draw's half word is compared in place: as the upper half of a word whose lower half can only add
// less than one, or shifted there; `threshold` stands in the upper half too.
struct Kept {
    bool at[8];
};
__device__ __forceinline__ Kept kept8(const HopMask& m, uint32_t block, int64_t row) {
    uint32_t w[4];
    philox(m, block, row, w);
    Kept k;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        k.at[2 * i] = w[i] << 16 >= m.threshold;
        k.at[2 * i + 1] = w[i] >= m.threshold;
    }
    return k;
}

// A workgroup takes 256 / `across` rows side by side, `across` threads (a power of two) each.
template <typename T>
__global__ __launch_bounds__(256) void dropout_kernel(const T* x, int64_t ldx, T* y, int64_t ldy, int64_t rows, int cols, int log_across, HopMask m) {
    const int across = 1 << log_across, c = ((int)blockIdx.x * across + ((int)threadIdx.x & (across - 1))) * 8, n = min(cols - c, 8);
    if (n <= 0) return;
    const int64_t step = (int64_t)gridDim.y * (256 >> log_across);
    for (int64_t r = (int64_t)blockIdx.y * (256 >> log_across) + (threadIdx.x >> log_across); r < rows; r += step) {
        const f32x8 v = wide<T>(columns8(x + r * ldx, cols, (uint32_t)c * (uint32_t)sizeof(T), n)) * m.factor;
        f32x8 to = 0.f;
        if (!m.none) {
            const Kept k = kept8(m, (uint32_t)c >> 3, m.first_row + r);
#pragma unroll
            for (int i = 0; i < 8; ++i) to[i] = k.at[i] ? v[i] : 0.f;
        }
        put8(y + r * ldy, (uint32_t)c * (uint32_t)sizeof(T), n, to);
    }
}

// ---- sums over a row ----------------------------------------------------------------
// Sum over a wavefront, the same bits in every lane: pairs, quads, halves and rows of 16 by DPP, rows joined by its broadcasts (a shuffle
// goes through LDS, six times over).
template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp_add(float v) {
    return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, ROWS, 0xF, false));
}
__device__ __forceinline__ float wave_sum(float v) {
    v = dpp_add<0xB1, 0xF>(v);          // quad_perm 1 0 3 2
    v = dpp_add<0x4E, 0xF>(v);          // quad_perm 2 3 0 1
    v = dpp_add<0x141, 0xF>(v);         // row_half_mirror
    v = dpp_add<0x140, 0xF>(v);         // row_mirror
    v = dpp_add<0x142, 0xA>(v);         // row_bcast 15 into rows 1 and 3
    v = dpp_add<0x143, 0xC>(v);         // row_bcast 31 into rows 2 and 3
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}

// One or two sums over the workgroup's threads, the same bits in every thread.  One barrier: the wavefronts' parts alternate between
// two places, and whoever writes a place again has passed the barrier behind the sum in between.
template <int NT>
struct RowSums {
    float* s;                                   // LDS: 2 x 2 x NT / 64
    int turn;
    __device__ __forceinline__ void operator()(float& a, float& b) {
        a = wave_sum(a);
        b = wave_sum(b);
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
        a = wave_sum(a);
        if (NT == 64) return;
        constexpr int W = NT / 64;
        float* p = s + turn * 2 * W;
        turn ^= 1;
        if ((threadIdx.x & 63) == 0) p[threadIdx.x >> 6] = a;
        __syncthreads();
        a = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) a += p[w];
    }
};
__device__ __forceinline__ float sum8(f32x8 v) { return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7])); }
__device__ __forceinline__ float dot8(f32x8 v, f32x8 w, float a) {
    float b = v[1] * w[1];
    a = fmaf(v[0], w[0], a);
    b = fmaf(v[3], w[3], b);
    a = fmaf(v[2], w[2], a);
    b = fmaf(v[5], w[5], b);
    a = fmaf(v[4], w[4], a);
    b = fmaf(v[7], w[7], b);
    a = fmaf(v[6], w[6], a);
    return a + b;
}
__device__ __forceinline__ float squares8(f32x8 v, float a) { return dot8(v, v, a); }
// v - mean in the n columns that exist, 0 elsewhere
__device__ __forceinline__ f32x8 centred(f32x8 v, float mean, int n) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? v[i] - mean : 0.f;
    return v;
}
// 1 / (1 + e^-z), e^-z as the unit's 2^t with t = -z log2(e).  For rows in 32 bits what rounding t loses is put back to first order - up to 64
// units of 2^-24 at z = -85 without it, 7 in all with it; rows in 16 bits keep 2^-9 of the result.  An infinite t leaves no finite rest, and any
// will do: e^-z is then 0 or infinite whatever it is multiplied with.
template <typename T>
__device__ __forceinline__ float logistic1(float z) {
    constexpr double kLog2 = 1.4426950408889634, kLn2 = 0.6931471805599453;
    constexpr float kLog2e = (float)kLog2, kLog2eRest = (float)(kLog2 - kLog2e);
    const float t = -z * kLog2e;
    float e = __builtin_amdgcn_exp2f(t);
    if constexpr (sizeof(T) == 4) {
        const float rest = fminf(fmaxf(fmaf(-z, kLog2eRest, fmaf(-z, kLog2e, -t)), -1.f), 1.f);
        e *= fmaf(rest, (float)kLn2, 1.f);
    }
    return __builtin_amdgcn_rcpf(1.f + e);
}
template <typename T>
__device__ __forceinline__ f32x8 logistic(f32x8 z) {
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = logistic1<T>(z[i]);
    return z;
}

// The vectors of a group that a workgroup needs for all its rows wait in LDS, each thread's own columns (so there is no barrier; in registers they
// would take the place of rows under way): two of them forwards, 8 bytes a column, three back, 12.  Kept for rows of up to 8192 columns, which are those
// whose next row is loaded ahead: beyond, 12 bytes a column are more than the LDS, and the registers do not hold even the one row (see launch).
template <int NT, int V>
struct Vectors {
    static constexpr bool kKept = NT * V <= 1024;
    f32x4 (*kept)[2 * V][kKept ? NT : 1];
    __device__ __forceinline__ void put(int w, int i, f32x8 v) const {
        kept[w][2 * i][threadIdx.x] = f32x4{v[0], v[1], v[2], v[3]};
        kept[w][2 * i + 1][threadIdx.x] = f32x4{v[4], v[5], v[6], v[7]};
    }
    __device__ __forceinline__ f32x8 get(int w, int i) const {
        const f32x4 a = kept[w][2 * i][threadIdx.x], b = kept[w][2 * i + 1][threadIdx.x];
        return f32x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    }
};

// A workgroup takes a piece of consecutive rows of one group, so the group's vectors are read once for all of them; the next
// row's loads are on their way while a row's statistics are worked out.
template <typename T, int NT, int V, bool EVEN>
__global__ __launch_bounds__(NT) void residual_kernel(HopResidualTask t, HopIndex index) {
    typedef Vectors<NT, V> Vec;
    __shared__ float shared[4 * (NT / 64)];
    __shared__ f32x4 kept[Vec::kKept ? 2 : 1][2 * V][Vec::kKept ? NT : 1];
    RowSums<NT> sums{shared, 0};
    const Vec vec{kept};
    int g, r0, r1;
    if (!find_piece(t.rows, t.shift, blockIdx.x, &g, &r0, &r1)) return;
    const int at = t.indexed ? index.at[g] : g;
    uint32_t col[V];
    int n[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        col[i] = (i * NT + threadIdx.x) * 8;
        n[i] = min(t.cols - (int)col[i], 8);
    }
    auto global = [&](const float* p, int64_t stride, int i) {
        return p ? columns8(p + at * stride, t.cols, col[i] * 4, n[i]) : f32x8(1.f);
    };
    // all that the branch is multiplied with beside its norm and the element's gate
    const float factor = t.scale * t.mask.factor;
    auto global_branch = [&](int i) { return global(t.post, t.post_stride, i) * (t.gate ? global(t.gate, t.gate_stride, i) * factor : f32x8(factor)); };
    if constexpr (Vec::kKept) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            vec.put(0, i, global_branch(i));
            vec.put(1, i, global(t.pre, t.pre_stride, i));
        }
    }
    typedef Matrix<T, EVEN> M;
    const M mx(t.x, t.ldx, t.cols), mb(t.b, t.ldb, t.cols), mz(t.z, t.ldz, t.cols), my(t.y, t.ldy, t.cols), mh(t.h, t.ldh, t.cols);
    raw_of<T> nx[V], nb[V], nz[V];
    auto fetch = [&](int r) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            nx[i] = mx.load(r, col[i], n[i]);
            nb[i] = mb.load(r, col[i], n[i]);
            nz[i] = mz.load(r, col[i], n[i]);
        }
    };
    constexpr bool kAhead = NT * V <= 1024;
    if (kAhead) fetch(r0);
    for (int r = r0; r < r1; ++r) {
        if (!kAhead) fetch(r);
        f32x8 x[V], b[V];
        raw_of<T> z[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            x[i] = wide<T>(nx[i]);
            b[i] = wide<T>(nb[i]);
            z[i] = nz[i];
        }
        if (kAhead && r + 1 < r1) fetch(r + 1);
        if (t.b) {
            float factor_b = 1.f;
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
                for (int i = 0; i < V; ++i) a = squares8(b[i], a);
                sums(a);
                factor_b = rsqrtf(a * t.inv_cols + t.eps);
            }
#pragma unroll
            for (int i = 0; i < V; ++i) {
                f32x8 u = b[i];
                if constexpr (Vec::kKept) u *= vec.get(0, i);
                else u *= global_branch(i);
                if (t.z) u *= logistic<T>(wide<T>(z[i]));
                if (t.mask.threshold) {
                    if (!t.mask.none) {
                        const Kept k = kept8(t.mask, col[i] >> 3, t.mask.first_row + r);
#pragma unroll
                        for (int j = 0; j < 8; ++j) x[i][j] = k.at[j] ? fmaf(u[j], factor_b, x[i][j]) : x[i][j];
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[i][j] = fmaf(u[j], factor_b, x[i][j]);
                }
                my.store(r, col[i], n[i], x[i]);
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
            for (int i = 0; i < V; ++i) a = squares8(x[i], a);
            sums(a);
            a = rsqrtf(a * t.inv_cols + t.eps);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                f32x8 pre;
                if constexpr (Vec::kKept) pre = vec.get(1, i);
                else pre = global(t.pre, t.pre_stride, i);
                mh.store(r, col[i], n[i], x[i] * a * pre);
            }
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
    for (int i = 0; i < V; ++i) a = squares8(v[i], a);
    sums(a);
    *r = rsqrtf(a * inv_cols + eps);
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] *= *r;
}
// a <- r (a - [mean a] - n mean(a n)): the gradient through a norm whose result was n; 0 in columns that do not exist
template <int NT, int V>
__device__ __forceinline__ void through_norm(f32x8 (&a)[V], const f32x8 (&nv)[V], const int (&n)[V], int norm, float inv_cols, float r, RowSums<NT>& sums) {
    float sn = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) sn = dot8(a[i], nv[i], sn);
    if (norm == HOP_NORM_CENTRED) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) s += sum8(a[i]);
        sums(s, sn);
#pragma unroll
        for (int i = 0; i < V; ++i) a[i] = centred(a[i], s * inv_cols, n[i]);
    } else {
        sums(sn);
    }
    sn *= -inv_cols * r;
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) a[i][j] = fmaf(nv[i][j], sn, a[i][j] * r);
}

// As in the forward pass; the parameters' gradients are summed over the piece's rows in registers and leave once a piece (with the group's
// vectors in registers too, 512 threads would fit a CU once, not twice).  Z: the gate is a tensor.
template <typename T, int NT, int V, bool EVEN, bool Z>
__global__ __launch_bounds__(NT) void residual_grad_kernel(HopResidualTask t, HopIndex index) {
    typedef Vectors<NT, V> Vec;
    constexpr bool kAhead = NT * V <= 1024;
    __shared__ float shared[4 * (NT / 64)];
    __shared__ f32x4 kept[Vec::kKept ? 3 : 1][2 * V][Vec::kKept ? NT : 1];
    RowSums<NT> sums{shared, 0};
    const Vec vec{kept};
    int g, r0, r1;
    if (!find_piece(t.rows, t.shift, blockIdx.x, &g, &r0, &r1)) return;
    const int at = t.indexed ? index.at[g] : g;
    uint32_t col[V];
    int n[V];
    f32x8 dpost[V] = {}, dpre[V] = {}, dgate[V] = {};
#pragma unroll
    for (int i = 0; i < V; ++i) {
        col[i] = (i * NT + threadIdx.x) * 8;
        n[i] = min(t.cols - (int)col[i], 8);
    }
    auto global = [&](const float* p, int64_t stride, int i) {
        return p ? columns8(p + at * stride, t.cols, col[i] * 4, n[i]) : f32x8(1.f);
    };
    auto read = [&](int w, int i) {
        return w == 0 ? global(t.post, t.post_stride, i) : w == 1 ? global(t.pre, t.pre_stride, i) : global(t.gate, t.gate_stride, i);
    };
    if constexpr (Vec::kKept) {
#pragma unroll
        for (int w = 0; w < 3; ++w)
#pragma unroll
            for (int i = 0; i < V; ++i) vec.put(w, i, read(w, i));
    }
    auto vector = [&](int w, int i) {
        if constexpr (Vec::kKept) return vec.get(w, i);
        else return read(w, i);
    };
    typedef Matrix<T, EVEN> M;
    const M mdy(t.dy, t.lddy, t.cols), mdh(t.dh, t.lddh, t.cols), my(t.dh ? t.y : nullptr, t.ldy, t.cols), mb(t.b, t.ldb, t.cols), mz(t.z, t.ldz, t.cols);
    const M mdx(t.dx, t.lddx, t.cols), mdb(t.db, t.lddb, t.cols), mdz(t.dz, t.lddz, t.cols);
    raw_of<T> next_dy[V], next_dh[V], next_y[V], next_b[V], next_z[V];
    auto fetch = [&](int r) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            next_dy[i] = mdy.load(r, col[i], n[i]);
            next_dh[i] = mdh.load(r, col[i], n[i]);
            next_y[i] = my.load(r, col[i], n[i]);
            next_b[i] = mb.load(r, col[i], n[i]);
            if (Z) next_z[i] = mz.load(r, col[i], n[i]);
        }
    };
    if (kAhead) fetch(r0);
    for (int r = r0; r < r1; ++r) {
        f32x8 e[V], a[V], v[V], b[V];
        raw_of<T> z[V];
        if (!kAhead) fetch(r);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            e[i] = wide<T>(next_dy[i]);
            a[i] = wide<T>(next_dh[i]);
            v[i] = wide<T>(next_y[i]);
            b[i] = wide<T>(next_b[i]);
            if (Z) z[i] = next_z[i];
        }
        if (kAhead && r + 1 < r1) fetch(r + 1);
        if (t.dh) {
            float f;
            normalise<NT, V>(v, n, t.next_norm, t.inv_cols, t.eps, &f, sums);
#pragma unroll
            for (int i = 0; i < V; ++i) {
#pragma unroll
                for (int j = 0; j < 8; ++j) dpre[i][j] = fmaf(a[i][j], v[i][j], dpre[i][j]);
                a[i] *= vector(1, i);
            }
            through_norm<NT, V>(a, v, n, t.next_norm, t.inv_cols, f, sums);
#pragma unroll
            for (int i = 0; i < V; ++i) e[i] += a[i];
        }
#pragma unroll
        for (int i = 0; i < V; ++i) mdx.store(r, col[i], n[i], e[i]);
        if (!t.b) continue;
        float rb = 1.f;
        if (t.norm) normalise<NT, V>(b, n, t.norm, t.inv_cols, t.eps, &rb, sums);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            f32x8 f = e[i] * (t.scale * t.mask.factor);
            if (t.mask.none) {
                f = f32x8(0.f);
            } else if (t.mask.threshold) {
                const Kept k = kept8(t.mask, col[i] >> 3, t.mask.first_row + r);
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = k.at[j] ? f[j] : 0.f;
            }
            const f32x8 post = vector(0, i), fn = f * b[i];
            if (Z) {
                const f32x8 s = logistic<T>(wide<T>(z[i])), fs = fn * s;
                mdz.store(r, col[i], n[i], fs * post * (1.f - s));
                dpost[i] += fs;
                a[i] = f * s * post;
            } else if (t.gate) {
                const f32x8 gate = vector(2, i);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    dgate[i][j] = fmaf(fn[j], post[j], dgate[i][j]);
                    dpost[i][j] = fmaf(fn[j], gate[j], dpost[i][j]);
                }
                a[i] = f * gate * post;
            } else {
                dpost[i] += fn;
                a[i] = f * post;
            }
        }
        if (t.db) {
            if (t.norm) through_norm<NT, V>(a, b, n, t.norm, t.inv_cols, rb, sums);
#pragma unroll
            for (int i = 0; i < V; ++i) mdb.store(r, col[i], n[i], a[i]);
        }
    }
    if (!t.partial) return;
    float* p = t.partial + (int64_t)blockIdx.x * 3 * t.cols;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if (n[i] <= 0) continue;
        if (t.dpost) put8(p, col[i] * 4, n[i], dpost[i]);
        if (t.dpre) put8(p + t.cols, col[i] * 4, n[i], dpre[i]);
        if (t.dgate) put8(p + 2 * (int64_t)t.cols, col[i] * 4, n[i], dgate[i]);
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

int64_t threads_for(int64_t cols) { return cols <= 512 ? 64 : cols <= 1024 ? 128 : cols <= 2048 ? 256 : 512; }
// Rows of a piece, as a power of two: as many as leave `pieces` of them.
int shift_for(int64_t rows, int64_t pieces) {
    int shift = 0;
    while ((shift < 7 && (rows >> (shift + 1)) >= pieces) || (rows >> shift) > 1 << 18) ++shift;
    return shift;
}

int64_t pieces_of(int64_t rows, int G, int shift) { return (rows >> shift) + (G < rows ? G : rows); }

template <typename T, int NT, int V, bool EVEN, bool GRAD>
void launch(const HopResidualTask& t, const HopIndex& index, int64_t pieces, hipStream_t st) {
    const dim3 grid((unsigned)pieces);
    if constexpr (!GRAD) residual_kernel<T, NT, V, EVEN><<<grid, NT, 0, st>>>(t, index);
    else if (t.z) residual_grad_kernel<T, NT, V, EVEN, true><<<grid, NT, 0, st>>>(t, index);
    else residual_grad_kernel<T, NT, V, EVEN, false><<<grid, NT, 0, st>>>(t, index);
}
template <typename T, bool EVEN, bool GRAD>
void launch(const HopResidualTask& t, const HopIndex& index, int64_t pieces, hipStream_t st) {
    // 1024 threads leave a gradient in 32 bits short of registers (4096 x 8192 with a gate for every element: 265 us, 234 with 512 threads of twice
    // eight columns; without gate 180 both ways, 7001 columns 199 and 210)
    constexpr int kTwice = GRAD && sizeof(T) == 4 ? 2 : 1;
    if (t.cols <= 512) launch<T, 64, 1, EVEN, GRAD>(t, index, pieces, st);
    else if (t.cols <= 1024) launch<T, 128, 1, EVEN, GRAD>(t, index, pieces, st);
    else if (t.cols <= 2048) launch<T, 256, 1, EVEN, GRAD>(t, index, pieces, st);
    else if (t.cols <= 4096) launch<T, 512, 1, EVEN, GRAD>(t, index, pieces, st);
    else if (t.cols <= 6144) launch<T, 768, 1, EVEN, GRAD>(t, index, pieces, st);
    else if (t.cols <= 8192) launch<T, 1024 / kTwice, kTwice, EVEN, GRAD>(t, index, pieces, st);
    else if (t.cols <= 16384) launch<T, 1024, 2, EVEN, GRAD>(t, index, pieces, st);
    else launch<T, 1024, 4, EVEN, GRAD>(t, index, pieces, st);
}
template <typename T, bool GRAD>
void launch(const HopResidualTask& t, const HopIndex& index, int64_t pieces, hipStream_t st) {
    // buffer accesses want addresses that are multiples of four
    auto even = [](const void* p, int64_t ld) { return ((uintptr_t)p & 3u) == 0 && (!p || ld * (int64_t)sizeof(T) % 4 == 0); };
    const bool all = t.cols % 8 == 0 && even(t.x, t.ldx) && even(t.b, t.ldb) && even(t.z, t.ldz) && even(t.y, t.ldy) && even(t.h, t.ldh) &&
                     even(t.dy, t.lddy) && even(t.dh, t.lddh) && even(t.dx, t.lddx) && even(t.db, t.lddb) && even(t.dz, t.lddz);
    if (all) launch<T, true, GRAD>(t, index, pieces, st);
    else launch<T, false, GRAD>(t, index, pieces, st);
}

}  // namespace

int hopl_dropout(int dtype, const void* x, int64_t ldx, void* y, int64_t ldy, int64_t rows, int64_t cols, const HopMask& m, void* stream) {
    hipStream_t st = (hipStream_t)stream;
    int log_across = 0;
    while (log_across < 8 && 8 << log_across < cols) ++log_across;
    const int64_t blocks = (rows + (256 >> log_across) - 1) >> (8 - log_across);
    const dim3 grid((unsigned)((cols + (8 << log_across) - 1) >> (3 + log_across)), (unsigned)(blocks < 65535 ? blocks : 65535));
    if (dtype == HOP_BF16) dropout_kernel<bf16><<<grid, 256, 0, st>>>((const bf16*)x, ldx, (bf16*)y, ldy, rows, (int)cols, log_across, m);
    else dropout_kernel<float><<<grid, 256, 0, st>>>((const float*)x, ldx, (float*)y, ldy, rows, (int)cols, log_across, m);
    return (int)hipGetLastError();
}

int hopl_residual(HopResidualTask t, int dtype, const HopIndex& index, void* stream) {
    // several workgroups a CU, and where registers leave room for one or two, as many pieces as that (16384 x 4096 in bf16: 4096 pieces 105 us,
    // 256 113, 16384 151)
    t.shift = shift_for(t.rows.rows, t.cols <= 4096 ? 256 * 4096 / threads_for(t.cols) : 256);
    const int64_t pieces = pieces_of(t.rows.rows, t.rows.G, t.shift);
    if (dtype == HOP_BF16) launch<bf16, false>(t, index, pieces, (hipStream_t)stream);
    else launch<float, false>(t, index, pieces, (hipStream_t)stream);
    return (int)hipGetLastError();
}

// Gradient: a piece's sums have to be joined with the others', so few rows go in few pieces too.  At least 768 pieces of up to 1024 columns (bf16,
// 16384 x 1024: 2048 pieces 84 us, 1024 65, 512 80; with fewer rows half as many would do: 4096 x 1024 39 and 35 us, 1000 x 256 with 1000 28,
// with 250 17), 256 of up to 2048 (512 x 2048: 512 pieces 26 us, 256 19, 128 19; 16384: 1024 111, 512 100, 256 131), 192 beyond (777 x 5001 with
// its 194 pieces 36 us, 388 45, 97 50; 16384 x 4096: 1024 pieces 206 us, 512 183, 256 170, 128 275).
int hopl_grad_shift(int64_t rows, int64_t cols) {
    return shift_for(rows, cols <= 1024 ? 768 : cols <= 2048 ? 256 : 192);
}
int64_t hopl_grad_chunks(int64_t rows, int G, int64_t cols) { return pieces_of(rows, G, hopl_grad_shift(rows, cols)); }

int hopl_residual_grad(HopResidualTask t, int dtype, const HopIndex& index, const HopIndex& dindex, void* stream) {
    hipStream_t st = (hipStream_t)stream;
    t.shift = hopl_grad_shift(t.rows.rows, t.cols);
    const int64_t chunks = pieces_of(t.rows.rows, t.rows.G, t.shift);
    if (chunks > 0) {
        if (dtype == HOP_BF16) launch<bf16, true>(t, index, chunks, st);
        else launch<float, true>(t, index, chunks, st);
    }
    if (t.dpost || t.dpre || t.dgate) {
        const dim3 grid((unsigned)((t.cols + 63) / 64), (unsigned)t.rows.G, 3);
        if (chunks / t.rows.G > 32 && grid.x * grid.y < 512) residual_join_kernel<16><<<grid, 1024, 0, st>>>(t, (int)chunks, dindex);
        else residual_join_kernel<4><<<grid, 256, 0, st>>>(t, (int)chunks, dindex);
    }
    return (int)hipGetLastError();
}
