// Gradients of softmax attention (hop_attention.hip), for gfx950 (CDNA4).
//
//   p_ij = exp(scale q_i k_j - lse_i),  D_i = sum_c do_ic o_ic,  ds_ij = p_ij (do_i v_j - D_i)
//   dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i,  dv_j = sum_i p_ij do_i              10 pairs cols operations
//
// Two kernels, each with sums of its own in registers, so that nothing is added up in memory and results are the same bits every time: one passes over the keys of a run of
// pairs for dq (and leaves D and lse for the other), one over the pairs of a run of keys for dk and dv.  The price is that scores and do v^T are
// computed twice: 14 operations where 10 would do.
#include <algorithm>
#include <type_traits>

#include "hop_attention_device.h"

using namespace hopa;

namespace {

template <typename T, int D>
constexpr int kTileRows = D * (int)sizeof(T) <= 256 ? 64 : 32;

__device__ __forceinline__ int64_t pairs_of(const HopAttentionTask& t) { return (int64_t)t.q_rows * t.group; }

// ---- dq ---------------------------------------------------------------------------------
template <typename T, int D, bool FED>
__global__ __launch_bounds__(256, sizeof(T) == 4 ? 1 : 2) void attention_dq_kernel(HopAttentionTask t) {
    typedef Tile<T, D> L;
    constexpr int NT = 256, kRows = kTileRows<T, D>, kBytes = kRows * L::kLine, kU = D / 32, kShift = 7;
    __shared__ __attribute__((aligned(16))) char sk0[kBytes], sv0[kBytes], sk1[kBytes], sv1[kBytes];
    const int head = blockIdx.x % t.k_heads, rest = blockIdx.x / t.k_heads, part = rest % t.parts;
    int s, first;
    if (!find_tile(t.q_begin, t.S, t.q_rows, t.group, kShift, true, rest / t.parts, &s, &first)) return;
    const Sequence seq = sequence(t, s);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, hi = lane >> 5;
    const int pairs = seq.nq * t.group, mine = first + wave * 32, pair = mine + (lane & 31);
    const bool live = pair < pairs;
    const int row = live ? divide(pair, t.group_inverse) : 0, its = live ? pair - row * t.group : 0;
    const int64_t at = seq.q0 + row;
    const int column = (head * t.group + its) * t.cols;
    const T* k = (const T*)t.k + seq.k0 * t.ldk + head * t.cols;
    const T* v = (const T*)t.v + seq.k0 * t.ldv + head * t.cols;

    typename L::frag fq[L::kSteps], fg[L::kSteps];
    load_columns<T, D, FED>(fq, (const T*)t.q + at * t.ldq + column, t.cols, live);
    load_columns<T, D, FED>(fg, (const T*)t.grad + at * t.ldgrad + column, t.cols, live);
    float delta = 0.f;
    {
        typename L::frag fo[L::kSteps];
        load_columns<T, D, FED>(fo, (const T*)t.o + at * t.ldo + column, t.cols, live);
#pragma unroll
        for (int i = 0; i < L::kSteps; ++i)
#pragma unroll
            for (int e = 0; e < L::kChunk; ++e) delta = __builtin_fmaf((float)fo[i][e], (float)fg[i][e], delta);
    }
    delta = both_sum(delta);
    const float lse = live ? ((const HOPL_GLOBAL float*)t.lse)[(int64_t)(head * t.group + its) * t.q_rows + at] * (1.f / kLn2) : 0.f;
    if (live && !hi && part == 0) {
        HOPL_GLOBAL float* terms = (HOPL_GLOBAL float*)t.terms + head * pairs_of(t) + (int64_t)seq.q0 * t.group + pair;
        terms[0] = lse;
        terms[t.k_heads * pairs_of(t)] = delta;
    }
    const int limit = live ? visible(seq, t.causal, row) : seq.nk;
    auto visible_of = [&](int p) { return visible(seq, t.causal, divide(p, t.group_inverse)); };
    const int all_see = visible_of(mine), some_see = mine < pairs ? visible_of(min(mine + 32, pairs) - 1) : 0, all_see_here = visible_of(first);
    const int chunk = (seq.nk + t.parts - 1) / t.parts, whole = (chunk + kRows - 1) / kRows * kRows;
    const int64_t from = (int64_t)part * whole;
    const int begin = from < seq.nk ? (int)from : seq.nk;
    const int end = min(min(begin + whole, seq.nk), visible_of(min(first + (1 << kShift), pairs) - 1));

    const Rows gk = {t.ldk, 1, 0, t.cols}, gv = {t.ldv, 1, 0, t.cols};
    Feed<T, D, kRows, NT, FED, false> feed_k, feed_v;
    auto issue = [&](char* sk, char* sv, int key) __attribute__((always_inline)) {
        feed_k.issue(sk, k, gk, key, seq.nk - key);
        feed_v.issue(sv, v, gv, key, seq.nk - key);
    };
    auto put = [&](char* sk, char* sv) __attribute__((always_inline)) {
        feed_k.put(sk);
        feed_v.put(sv);
    };
    f32x16 dq[kU];
    auto turn = [&](const char* sk, const char* sv, int key) __attribute__((always_inline)) {
        if (key >= some_see) return;
#pragma unroll
        for (int u = 0; u < kRows / 32; ++u) {
            f32x16 p = (f32x16)(0.f), ds = (f32x16)(0.f);
#pragma unroll
            for (int i = 0; i < L::kSteps; ++i) {
                p = multiply(L::along(sk, 32 * u, i), fq[i], p);
                ds = multiply(L::along(sv, 32 * u, i), fg[i], ds);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) ds[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[r], t.scale_log2, -lse)) * (ds[r] - delta);
            if (key + 32 * u + 32 > all_see) {
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (key + 32 * u + 8 * (r >> 2) + 4 * hi + (r & 3) >= limit) ds[r] = 0.f;
            }
            const Weights<T> w(ds);
#pragma unroll
            for (int c = 0; c < kU; ++c) dq[c] = w.template product<D>(sk, 32 * u, c, dq[c]);
        }
    };
    auto pass = [&](auto careful) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < kU; ++c) dq[c] = (f32x16)(0.f);
        auto take = [&](char* sk, const char* sv, int key) __attribute__((always_inline)) {
            if constexpr (decltype(careful)::value) {
                if (key + kRows > all_see_here) {
                    add_not_finite<T, D>(sk, min(kRows, seq.nk - key), dq, [&](int j) { return key + j < limit; });
                    __syncthreads();
                    drop_not_finite<T, kBytes, NT>(sk);
                    __syncthreads();
                }
            }
            turn(sk, sv, key);
        };
        if (begin < end) {
            issue(sk0, sv0, begin);
            put(sk0, sv0);
        }
        for (int key = begin; key < end; key += 2 * kRows) {
            arrive();
            const bool second = key + kRows < end, third = key + 2 * kRows < end;
            if (second) issue(sk1, sv1, key + kRows);
            take(sk0, sv0, key);
            if (!second) break;
            put(sk1, sv1);
            arrive();
            if (third) issue(sk0, sv0, key + 2 * kRows);
            take(sk1, sv1, key + kRows);
            if (third) put(sk0, sv0);
        }
    };
    pass(std::false_type());
    if (t.causal && __syncthreads_or(live && !all_finite(dq))) pass(std::true_type());
    if (!live) return;
    if (t.parts > 1) {
        const int64_t to = ((int64_t)part * t.k_heads + head) * pairs_of(t) + (int64_t)seq.q0 * t.group + pair;
        store_columns<float, D>(t.partial + to * t.cols, t.cols, dq, 1.f);
    } else {
        store_columns<T, D>((T*)t.dq + at * t.lddq + column, t.cols, dq, t.scale);
    }
}

// ---- dk and dv ------------------------------------------------------------------------------
template <typename T, int D, bool FED>
__global__ __launch_bounds__(256, sizeof(T) == 4 ? 1 : 2) void attention_dkv_kernel(HopAttentionTask t) {
    typedef Tile<T, D> L;
    constexpr int NT = 256, kRows = kTileRows<T, D>, kBytes = kRows * L::kLine, kU = D / 32, kShift = 7;
    __shared__ __attribute__((aligned(16))) char sq0[kBytes], sg0[kBytes], sq1[kBytes], sg1[kBytes];
    __shared__ __attribute__((aligned(16))) float st0[128], st1[128];              // lse log2(e) of 64 pairs, then their D
    const int head = blockIdx.x % t.k_heads, rest = blockIdx.x / t.k_heads, part = rest % t.parts;
    int s, first;
    if (!find_tile(t.k_begin, t.S, t.k_rows, 1, kShift, false, rest / t.parts, &s, &first)) return;
    const Sequence seq = sequence(t, s);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, hi = lane >> 5;
    const int mine = first + wave * 32, key = mine + (lane & 31);
    const bool live = key < seq.nk;
    const int64_t at = seq.k0 + (live ? key : 0);
    const int pairs = seq.nq * t.group;
    const T* q = (const T*)t.q + seq.q0 * t.ldq + head * t.group * t.cols;
    const T* g = (const T*)t.grad + seq.q0 * t.ldgrad + head * t.group * t.cols;
    const float* terms = t.terms + head * pairs_of(t) + (int64_t)seq.q0 * t.group;

    typename L::frag fk[L::kSteps], fv[L::kSteps];
    load_columns<T, D, FED>(fk, (const T*)t.k + at * t.ldk + head * t.cols, t.cols, live);
    load_columns<T, D, FED>(fv, (const T*)t.v + at * t.ldv + head * t.cols, t.cols, live);
    auto seen_from = [&](int j) { return t.causal ? max(0, j - (seq.nk - seq.nq)) * t.group : 0; };        // the first pair that sees key j
    const int least = live ? seen_from(key) : 0;
    const int some_see = mine < seq.nk ? seen_from(mine) : pairs, all_see = seen_from(min(mine + 32, seq.nk) - 1);
    const int all_see_here = seen_from(min(first + (1 << kShift), seq.nk) - 1);
    const int start = seen_from(first) / kRows * kRows;
    const int chunk = (max(0, pairs - start) + t.parts - 1) / t.parts, whole = (chunk + kRows - 1) / kRows * kRows;
    const int64_t from = start + (int64_t)part * whole;
    const int begin = from < pairs ? (int)from : pairs, end = min(begin + whole, pairs);

    const Rows gq = {t.ldq, t.group, t.group_inverse, t.cols}, gg = {t.ldgrad, t.group, t.group_inverse, t.cols};
    Feed<T, D, kRows, NT, FED, true> feed_q, feed_g;
    auto issue = [&](char* sq, char* sg, float* st, int pair) __attribute__((always_inline)) {
        feed_q.issue(sq, q, gq, pair, pairs - pair);
        feed_g.issue(sg, g, gg, pair, pairs - pair);
        if (wave < 2) {
            const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)(terms + wave * t.k_heads * pairs_of(t) + pair), 0,
                                                                               min(kRows, pairs - pair) * 4, 0x00020000);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(st + wave * 64), 4, lane * 4, 0, 0, 0);
        }
    };
    auto put = [&](char* sq, char* sg) __attribute__((always_inline)) {
        feed_q.put(sq);
        feed_g.put(sg);
    };
    f32x16 dk[kU], dv[kU];
    auto turn = [&](const char* sq, const char* sg, const float* st, int pair) __attribute__((always_inline)) {
        if (pair + kRows <= some_see) return;
#pragma unroll
        for (int u = 0; u < kRows / 32; ++u) {
            f32x16 p = (f32x16)(0.f), ds = (f32x16)(0.f);
#pragma unroll
            for (int i = 0; i < L::kSteps; ++i) {
                p = multiply(L::along(sq, 32 * u, i), fk[i], p);
                ds = multiply(L::along(sg, 32 * u, i), fv[i], ds);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x4 lse = *(const f32x4*)(st + 32 * u + 8 * i + 4 * hi), delta = *(const f32x4*)(st + 64 + 32 * u + 8 * i + 4 * hi);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    p[4 * i + e] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[4 * i + e], t.scale_log2, -lse[e]));
                    ds[4 * i + e] = p[4 * i + e] * (ds[4 * i + e] - delta[e]);
                }
            }
            if (pair + 32 * u < all_see) {
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (pair + 32 * u + 8 * (r >> 2) + 4 * hi + (r & 3) < least) p[r] = ds[r] = 0.f;
            }
            const Weights<T> wp(p), ws(ds);
#pragma unroll
            for (int c = 0; c < kU; ++c) {
                dv[c] = wp.template product<D>(sg, 32 * u, c, dv[c]);
                dk[c] = ws.template product<D>(sq, 32 * u, c, dk[c]);
            }
        }
    };
    auto pass = [&](auto careful) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < kU; ++c) dk[c] = dv[c] = (f32x16)(0.f);
        auto take = [&](char* sq, char* sg, const float* st, int pair) __attribute__((always_inline)) {
            if constexpr (decltype(careful)::value) {
                if (pair < all_see_here) {
                    const int count = min(kRows, pairs - pair);
                    add_not_finite<T, D>(sq, count, dk, [&](int j) { return pair + j >= least; });
                    add_not_finite<T, D>(sg, count, dv, [&](int j) { return pair + j >= least; });
                    __syncthreads();
                    drop_not_finite<T, kBytes, NT>(sq);
                    drop_not_finite<T, kBytes, NT>(sg);
                    __syncthreads();
                }
            }
            turn(sq, sg, st, pair);
        };
        if (begin < end) {
            issue(sq0, sg0, st0, begin);
            put(sq0, sg0);
        }
        for (int pair = begin; pair < end; pair += 2 * kRows) {
            arrive();
            const bool second = pair + kRows < end, third = pair + 2 * kRows < end;
            if (second) issue(sq1, sg1, st1, pair + kRows);
            take(sq0, sg0, st0, pair);
            if (!second) break;
            put(sq1, sg1);
            arrive();
            if (third) issue(sq0, sg0, st0, pair + 2 * kRows);
            take(sq1, sg1, st1, pair + kRows);
            if (third) put(sq0, sg0);
        }
    };
    pass(std::false_type());
    if (t.causal && __syncthreads_or(live && !(all_finite(dk) && all_finite(dv)))) pass(std::true_type());
    if (!live) return;
    if (t.parts > 1) {
        const int64_t rows = t.k_rows, to = (((int64_t)part * 2 * t.k_heads + head) * rows + at) * t.cols;
        store_columns<float, D>(t.partial + to, t.cols, dk, 1.f);
        store_columns<float, D>(t.partial + to + t.k_heads * rows * t.cols, t.cols, dv, 1.f);
    } else {
        store_columns<T, D>((T*)t.dk + at * t.lddk + head * t.cols, t.cols, dk, t.scale);
        store_columns<T, D>((T*)t.dv + at * t.lddv + head * t.cols, t.cols, dv, 1.f);
    }
}

// ---- parts, joined in their order: a wavefront per row of a head -----------------------------------
__device__ __forceinline__ bool covered(const int32_t* begin, int S, int rows, int64_t row) {
    if (!begin) return row < rows;
    return row >= ((const HOPL_GLOBAL int32_t*)begin)[0] && row < ((const HOPL_GLOBAL int32_t*)begin)[S];
}
template <typename T>
__device__ __forceinline__ void join_row(const HopAttentionTask& t, int64_t at, int64_t next, T* to, float by) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int c = lane + 64 * i;
        if (c >= t.cols) continue;
        float v = 0.f;
        for (int p = 0; p < t.parts; ++p) v += ((const HOPL_GLOBAL float*)t.partial)[(at + p * next) * t.cols + c];
        ((HOPL_GLOBAL T*)to)[c] = (T)(v * by);
    }
}
template <typename T>
__global__ __launch_bounds__(256) void attention_dq_join_kernel(HopAttentionTask t) {
    const int64_t number = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), per_head = pairs_of(t);
    const int head = (int)(number / per_head);
    const int64_t pair = number - head * per_head, row = pair / t.group;
    if (head >= t.k_heads || !covered(t.q_begin, t.S, t.q_rows, row)) return;
    join_row<T>(t, head * per_head + pair, t.k_heads * per_head, (T*)t.dq + row * t.lddq + (head * t.group + (pair - row * t.group)) * t.cols, t.scale);
}
template <typename T>
__global__ __launch_bounds__(256) void attention_dkv_join_kernel(HopAttentionTask t) {
    const int64_t number = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int head = (int)(number / t.k_rows);
    const int64_t row = number - (int64_t)head * t.k_rows;
    if (head >= t.k_heads || !covered(t.k_begin, t.S, t.k_rows, row)) return;
    const int64_t at = (int64_t)head * t.k_rows + row, all = (int64_t)t.k_heads * t.k_rows;
    join_row<T>(t, at, 2 * all, (T*)t.dk + row * t.lddk + head * t.cols, t.scale);
    join_row<T>(t, at + all, 2 * all, (T*)t.dv + row * t.lddv + head * t.cols, 1.f);
}

template <typename T, int D, bool FED>
int launch(HopAttentionTask t, int dq_parts, int dkv_parts, hipStream_t stream) {
    const int64_t pairs = (int64_t)t.q_rows * t.group;
    hipError_t e = hipSuccess;
    if (t.q_rows) {
        t.parts = dq_parts;
        attention_dq_kernel<T, D, FED><<<dim3((unsigned)(((pairs + 127) / 128 + t.S) * t.k_heads * t.parts)), dim3(256), 0, stream>>>(t);
        if (t.parts > 1) attention_dq_join_kernel<T><<<dim3((unsigned)((pairs * t.k_heads + 3) / 4)), dim3(256), 0, stream>>>(t);
        e = hipGetLastError();
    }
    if (e == hipSuccess && t.k_rows) {
        t.parts = dkv_parts;
        attention_dkv_kernel<T, D, FED><<<dim3((unsigned)((((int64_t)t.k_rows + 127) / 128 + t.S) * t.k_heads * t.parts)), dim3(256), 0, stream>>>(t);
        if (t.parts > 1) attention_dkv_join_kernel<T><<<dim3((unsigned)(((int64_t)t.k_rows * t.k_heads + 3) / 4)), dim3(256), 0, stream>>>(t);
        e = hipGetLastError();
    }
    return (int)e;
}

template <typename T>
int launch(const HopAttentionTask& t, int dq_parts, int dkv_parts, hipStream_t stream) {
    auto fits = [&](const void* p, int64_t ld) { return ((uintptr_t)p & 15u) == 0 && (ld * sizeof(T)) % 16 == 0; };
    const bool fed = fits(t.q, t.ldq) && fits(t.k, t.ldk) && fits(t.v, t.ldv) && fits(t.grad, t.ldgrad) && fits(t.o, t.ldo) && (t.cols * sizeof(T)) % 16 == 0;
    if (t.cols <= 64) return fed ? launch<T, 64, true>(t, dq_parts, dkv_parts, stream) : launch<T, 64, false>(t, dq_parts, dkv_parts, stream);
    return fed ? launch<T, 128, true>(t, dq_parts, dkv_parts, stream) : launch<T, 128, false>(t, dq_parts, dkv_parts, stream);
}

int parts_of(int64_t tiles, int64_t length) { return (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>((512 + tiles - 1) / tiles, length / 256), 64)); }

}  // namespace

int hopa_dq_parts(const HopAttentionTask& t, int dtype) {
    (void)dtype;
    return parts_of((((int64_t)t.q_rows * t.group + 127) / 128 + t.S) * t.k_heads, t.k_rows / t.S);
}
int hopa_dkv_parts(const HopAttentionTask& t, int dtype) {
    (void)dtype;
    return parts_of((((int64_t)t.k_rows + 127) / 128 + t.S) * t.k_heads, (int64_t)t.q_rows * t.group / t.S);
}

int hopa_grad(const HopAttentionTask& t, int dtype, int dq_parts, int dkv_parts, void* stream) {
    return dtype == HOP_BF16 ? launch<bf16>(t, dq_parts, dkv_parts, (hipStream_t)stream) : launch<float>(t, dq_parts, dkv_parts, (hipStream_t)stream);
}
