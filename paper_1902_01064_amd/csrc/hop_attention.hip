// Softmax attention of packed sequences with grouped heads, for gfx950 (CDNA4).
//
//   o_i = sum_j p_ij v_j,  p_ij = exp(scale q_i k_j - lse_i),  lse_i = log sum_j exp(scale q_i k_j)     4 pairs cols operations
//
// A workgroup takes a run of a key head's pairs (query row, head of the group) and passes once over the keys that they see, tile by tile: scores
// keys x pairs on the matrix unit, their running maximum and sum column by column, and the product of the values with the softmax's terms, which never
// leave the registers.
//
// With many queries the matrix unit bounds it, and the exponentials beside it: 8192 tokens that all see each other, 16 heads of 128 columns on 2, bfloat16, take 525 us, 1047
// TFLOP/s; 53 % of the cycles have a product under way (writing down an order of products and exponentials within a wavefront changed nothing: two wavefronts to a SIMD fill each
// other's gaps).  With few, the keys' and values' bytes: 16 sequences of 16384 tokens in 206 us, 5.2 TB/s.
#include <algorithm>
#include <type_traits>

#include "hop_attention_device.h"

using namespace hopa;

namespace {

template <typename T, int D>
constexpr int kTileRows = D * (int)sizeof(T) <= 256 ? 64 : 32;


// What a part of the keys leaves for each pair: an unnormalised sum, and the maximum (in powers of two) and the sum of its terms.
__device__ __forceinline__ int64_t part_place(const HopAttentionTask& t, int part, int head, int64_t pair) {
    return ((int64_t)part * t.k_heads + head) * ((int64_t)t.q_rows * t.group) + pair;
}

// FEW: the wavefronts of a workgroup have the same 32 pairs and every so many stages of the keys each, buffers of their own, and no barrier before they add up what they have.
// One wavefront alone fetches keys no faster, and as parts of a launch they would need another one to be joined: 4 sequences of 500
// keys 14.3 us a call, now 10.3; 131072 keys of one 79, now 44.
template <typename T, int D>
constexpr int kFewRows = D * (int)sizeof(T) >= 256 ? 32 : 64;
template <typename T, int D>
constexpr int kFewWaves = 32768 / (kFewRows<T, D> * D * (int)sizeof(T));

template <typename T, int D, bool FED, bool FEW>
__global__ __launch_bounds__((FEW ? kFewWaves<T, D> : 4) * 64, (FEW || (sizeof(T) == 4 && D > 64) ? 1 : 2)) void attention_kernel(HopAttentionTask t) {
    typedef Tile<T, D> L;
    constexpr int kWaves = FEW ? kFewWaves<T, D> : 4, NT = FEW ? 64 : kWaves * 64;           // threads that fill a tile
    constexpr int kRows = FEW ? kFewRows<T, D> : kTileRows<T, D>, kBytes = kRows * L::kLine, kU = D / 32, kStep = (FEW ? kWaves : 1) * kRows;
    constexpr int kShift = FEW ? 5 : 7, kAtOnce = sizeof(T) == 4 ? kRows / 32 : 1;
    // arrays of their own, so that the compiler knows that reads of one stage need not wait for loads into the other
    constexpr int kAll = (FEW ? kWaves : 1) * kBytes;
    __shared__ __attribute__((aligned(16))) char all_k0[kAll], all_v0[kAll], all_k1[kAll], all_v1[kAll];
    const int head = blockIdx.x % t.k_heads, rest = blockIdx.x / t.k_heads, part = rest % t.parts;
    int s, first;
    if (!find_tile(t.q_begin, t.S, t.q_rows, t.group, kShift, rest / t.parts, &s, &first)) return;
    const Sequence seq = sequence(t, s);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, hi = lane >> 5;
    const int pairs = seq.nq * t.group, mine = first + (FEW ? 0 : wave * 32);            // the wavefront's first pair
    const int own = FEW ? wave * kBytes : 0;
    char *const sk0 = all_k0 + own, *const sv0 = all_v0 + own, *const sk1 = all_k1 + own, *const sv1 = all_v1 + own;
    // with everyone who shares a buffer
    auto meet = [&]() __attribute__((always_inline)) {
        if constexpr (FEW) asm volatile("" ::: "memory");
        else __syncthreads();
    };
    auto arrive_here = [&]() __attribute__((always_inline)) {
        if constexpr (FEW) {
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_waitcnt(0x0070);         // vmcnt(0) lgkmcnt(0)
            asm volatile("" ::: "memory");
        } else {
            arrive();
        }
    };
    const int pair = mine + (lane & 31);
    const bool live = pair < pairs;
    const int row = live ? hopa_divide(pair, t.group_inverse, t.group_shift) : 0, its = live ? pair - row * t.group : 0;
    const int limit = live ? visible(seq, t.causal, row) : seq.nk;             // keys that the lane's column sees
    const T* q = (const T*)t.q + (seq.q0 + row) * t.ldq + (head * t.group + its) * t.head;
    const T* k = (const T*)t.k + seq.k0 * t.ldk + head * t.head;
    const T* v = (const T*)t.v + seq.k0 * t.ldv + head * t.head;
    typename L::frag fq[L::kSteps];
    load_columns<T, D, FED>(fq, q, t.head, live);
    auto visible_of = [&](int pair) { return visible(seq, t.causal, hopa_divide(pair, t.group_inverse, t.group_shift)); };
    const int all_see = visible_of(mine), some_see = mine < pairs ? visible_of(min(mine + 32, pairs) - 1) : 0;
    const int all_see_here = visible_of(first);                                       // of the workgroup's
    const int chunk = (seq.nk + t.parts - 1) / t.parts, whole = (chunk + kRows - 1) / kRows * kRows;
    const int64_t from = (int64_t)part * whole;
    const int part_begin = from < seq.nk ? (int)from : seq.nk, begin = part_begin + (FEW ? wave * kRows : 0);
    const int end = min(min(part_begin + whole, seq.nk), visible_of(min(first + (1 << kShift), pairs) - 1));

    const Rows gk = {t.ldk, 1, 0, 0, t.head}, gv = {t.ldv, 1, 0, 0, t.head};
    Feed<T, D, kRows, NT, FED, false> feed_k, feed_v;
    feed_k.begin(gk, 0);
    feed_v.begin(gv, 0);
    auto issue = [&](char* sk, char* sv, int key) __attribute__((always_inline)) {
        feed_k.issue(sk, k, gk, key, seq.nk - key);
        feed_v.issue(sv, v, gv, key, seq.nk - key);
    };
    auto put = [&](char* sk, char* sv) __attribute__((always_inline)) {
        feed_k.put(sk);
        feed_v.put(sv);
    };

    const Places<T, D> places;
    f32x16 o[kU];
    float top, sum;                            // of scores in powers of two; over the lane's own half of the column
    auto clear = [&]() __attribute__((always_inline)) {
        top = -kInf;
        sum = 0.f;
#pragma unroll
        for (int c = 0; c < kU; ++c) o[c] = (f32x16)(0.f);
    };
    // N units of 32 keys at once: what one waits for, another fills.  In fp32 (32 sequences of 128 rows: 26 us, one by one 33); operands of bfloat16 need the
    // registers for other things (a prompt of 8192 rows: 235 us, one by one 203).
    auto units = [&](auto n, const char* sk, const char* sv, int key) __attribute__((always_inline)) {
        constexpr int N = decltype(n)::value;
        const Places<T, D> at = places;
        f32x16 p[N];
#pragma unroll
        for (int u = 0; u < N; ++u) p[u] = (f32x16)(0.f);
#pragma unroll
        for (int i = 0; i < L::kSteps; ++i)
#pragma unroll
            for (int u = 0; u < N; ++u) p[u] = multiply(L::along(sk + 32 * u * L::kLine, at.along, i), fq[i], p[u]);
        if (key + 32 * N > all_see) {
            asm volatile("");                  // a branch, which few tiles take, and not selections that all of them make
#pragma unroll
            for (int u = 0; u < N; ++u)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (key + 32 * u + 8 * (r >> 2) + 4 * hi + (r & 3) >= limit) p[u][r] = -kInf;
        }
        // The maximum is moved only when a score exceeds it by a factor of 2^8: terms of up to that are as exact, and most tiles leave the sums alone.
        float most = p[0][0];
#pragma unroll
        for (int u = 0; u < N; ++u)
#pragma unroll
            for (int r = 0; r < 16; ++r) most = fmaxf(most, p[u][r]);
        if (__any(__builtin_fmaf(most, t.scale_log2, -8.f) > top)) {
            // only of columns with such a score, so that a row's bits do not depend on the rows beside it; in front of the first one there is nothing to scale but what
            // the second pass added by hand, which zero would turn into NaN
            const float its = both_max(most) * t.scale_log2, now = its - 8.f > top ? its : top;
            const float by = now == top || top == -kInf ? 1.f : __builtin_amdgcn_exp2f(top - now);
            top = now;
            sum *= by;
#pragma unroll
            for (int c = 0; c < kU; ++c)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[c][e] *= by;
        }
        const float base = top == -kInf ? 0.f : top;
        float more[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < N; ++u)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                p[u][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[u][r], t.scale_log2, -base));
                more[r & 3] += p[u][r];
            }
        sum += (more[0] + more[1]) + (more[2] + more[3]);
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const Weights<T> w(p[u]);
            Sums<T, D> sums;
            sums.begin(sv + 32 * u * L::kLine, at.across);
            sums.add(sv + 32 * u * L::kLine, at.across, w, o);
        }
    };
    auto turn = [&](const char* sk, const char* sv, int key) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kRows / 32; u += kAtOnce) {
            if (key + 32 * u >= some_see) break;
            if (kAtOnce > 1 && key + 32 * (u + 1) >= some_see) units(std::integral_constant<int, 1>(), sk + 32 * u * L::kLine, sv + 32 * u * L::kLine, key + 32 * u);
            else units(std::integral_constant<int, kAtOnce>(), sk + 32 * u * L::kLine, sv + 32 * u * L::kLine, key + 32 * u);
        }
    };
    clear();
    if (begin < end) {
        issue(sk0, sv0, begin);
        put(sk0, sv0);
    }
    for (int key = begin; key < end; key += 2 * kStep) {
        arrive_here();
        const bool second = key + kStep < end, third = key + 2 * kStep < end;
        if (second) issue(sk1, sv1, key + kStep);
        turn(sk0, sv0, key);
        if (!second) break;
        put(sk1, sv1);
        arrive_here();
        if (third) issue(sk0, sv0, key + 2 * kStep);
        turn(sk1, sv1, key + kStep);
        if (third) put(sk0, sv0);
    }
    if (t.causal) {
        const bool odd = live && !all_finite(o);
        if (FEW ? __any(odd) : __syncthreads_or(odd)) {
            clear();
            for (int key = begin; key < end; key += kStep) {
                issue(sk0, sv0, key);
                put(sk0, sv0);
                arrive_here();
                if (key + kRows > (FEW ? all_see : all_see_here)) {
                    add_not_finite<T, D, D>(sv0, 0, 0, min(kRows, seq.nk - key), o, [&](int j) { return key + j < limit; });
                    meet();
                    drop_not_finite<T, kBytes, NT>(sv0);
                    arrive_here();
                }
                turn(sk0, sv0, key);
                arrive_here();
            }
        }
    }
    if constexpr (FEW) {
        // The wavefronts' sums at the largest of their maxima, added in their order by the first one.
        __shared__ float tops[kWaves][64], sums[kWaves][64];
        tops[wave][lane] = top;
        __syncthreads();
        float most = -kInf;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) most = fmaxf(most, tops[w][lane]);
        const float by = top == -kInf ? 0.f : __builtin_amdgcn_exp2f(top - most);
        sums[wave][lane] = top == -kInf ? sum : sum * by;              // where it is not zero, NaN
        auto place = [&](int w, int c) __attribute__((always_inline)) {           // of unit c: the wavefront's own buffers, of which it needs no more than these two
            return (c * 4096 < kBytes ? all_k0 + w * kBytes + c * 4096 : all_v0 + w * kBytes + c * 4096 - kBytes) + lane * 16;
        };
        if (wave)
#pragma unroll
            for (int c = 0; c < kU; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    *(f32x4*)(place(wave, c) + e * 1024) = {o[c][4 * e] * by, o[c][4 * e + 1] * by, o[c][4 * e + 2] * by, o[c][4 * e + 3] * by};
        __syncthreads();
        if (wave) return;
        top = most;
        sum = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) sum += sums[w][lane];
#pragma unroll
        for (int c = 0; c < kU; ++c)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[c][e] *= by;
        for (int w = 1; w < kWaves; ++w)
#pragma unroll
            for (int c = 0; c < kU; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const f32x4 more = *(const f32x4*)(place(w, c) + e * 1024);
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[c][4 * e + i] += more[i];
                }
    }

    const float total = both_sum(sum), base = top == -kInf ? 0.f : top;
    if (!live) return;
    if (t.parts > 1) {
        const int64_t at = part_place(t, part, head, (int64_t)seq.q0 * t.group + pair), all = part_place(t, t.parts, 0, 0);
        store_columns<float, D>(t.partial + at * t.cols, t.cols, o, 1.f);
        if (!hi) {
            ((HOPL_GLOBAL float*)t.partial)[all * t.cols + 2 * at] = base;
            ((HOPL_GLOBAL float*)t.partial)[all * t.cols + 2 * at + 1] = total;
        }
        return;
    }
    const int column = (head * t.group + its) * t.cols;
    store_columns<T, D>((T*)t.o + (seq.q0 + row) * t.ldo + column, t.cols, o, total == 0.f ? 0.f : 1.f / total);
    if (t.lse && !hi)
        ((HOPL_GLOBAL float*)t.lse)[(int64_t)(head * t.group + its) * t.q_rows + seq.q0 + row] =
            total == 0.f ? -kInf : (base + __builtin_amdgcn_logf(total)) * kLn2;
}

// Joins the parts in their order: a wavefront per pair, all parts' maxima at once.
template <typename T>
__global__ __launch_bounds__(256) void attention_join_kernel(HopAttentionTask t) {
    const int lane = threadIdx.x & 63;
    const int64_t all = part_place(t, t.parts, 0, 0);
    const uint32_t number = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), per_head = t.q_rows * t.group;          // below 2^30 in all
    const int head = number / per_head, pair = number - head * per_head, row = hopa_divide(pair, t.group_inverse, t.group_shift), its = pair - row * t.group;
    if (head >= t.k_heads) return;
    int b = 0, e = t.q_rows;
    if (t.q_begin) {
        b = ((const HOPL_GLOBAL int32_t*)t.q_begin)[0];
        e = ((const HOPL_GLOBAL int32_t*)t.q_begin)[t.S];
    }
    if (row < b || row >= e) return;
    const HOPL_GLOBAL float* sums = (const HOPL_GLOBAL float*)t.partial;
    const HOPL_GLOBAL float* tops = sums + all * t.cols;
    // a lane a part, of which there are 64 at most
    float its_top = -kInf, its_total = 0.f;
    if (lane < t.parts) {
        const int64_t at = part_place(t, lane, head, pair);
        its_total = tops[2 * at + 1];
        if (its_total != 0.f) its_top = tops[2 * at];
    }
    float top = its_top;
#pragma unroll
    for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    const float weight = its_total == 0.f ? 0.f : __builtin_amdgcn_exp2f(its_top - top);
    float total = weight * its_total, v[2] = {0.f, 0.f};
#pragma unroll
    for (int o = 32; o; o >>= 1) total += __shfl_xor(total, o);
#pragma unroll 4
    for (int p = 0; p < t.parts; ++p) {
        const float w = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(weight), p));
        const int64_t at = part_place(t, p, head, pair);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float x = lane + 64 * i < t.cols && w != 0.f ? sums[at * t.cols + lane + 64 * i] : 0.f;
            v[i] = __builtin_fmaf(w, x, v[i]);
        }
    }
    const float by = total == 0.f ? 0.f : 1.f / total;
    const int h = head * t.group + its;
    HOPL_GLOBAL T* o = (HOPL_GLOBAL T*)t.o + row * t.ldo + (int64_t)h * t.cols;
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (lane + 64 * i < t.cols) o[lane + 64 * i] = (T)(v[i] * by);
    if (t.lse && lane == 0) ((HOPL_GLOBAL float*)t.lse)[(int64_t)h * t.q_rows + row] = total == 0.f ? -kInf : (top + __builtin_amdgcn_logf(total)) * kLn2;
}

// Few pairs to a sequence.
bool few(const HopAttentionTask& t) { return (int64_t)t.q_rows * t.group <= (int64_t)32 * t.S; }

// Few queries read a key once, and that is all their time: they fill tiles from rows that are not aligned through registers, and others' rows are copied first.
// In fp32 tiles of 128 columns and what is on its way to them are more than all registers (172 bytes of scratch a lane), so there rows are copied for few queries too: the next token
// of 16 sequences of 8192 tokens, 8 key heads of 128 columns, 361 us, not aligned 793.  In bfloat16 twice as many tokens take 207 us, not aligned, through registers, 248.
template <typename T, int D>
constexpr bool kThroughRegisters = D * (int)sizeof(T) <= 256;

template <typename T, int D>
int launch(const HopAttentionTask& t, bool fed, hipStream_t stream) {
    const int64_t pairs = (int64_t)t.q_rows * t.group;
    if (few(t)) {
        const dim3 grid((unsigned)(((pairs + 31) / 32 + t.S) * t.k_heads * t.parts)), threads(kFewWaves<T, D> * 64);
        if constexpr (kThroughRegisters<T, D>) {
            if (fed) attention_kernel<T, D, true, true><<<grid, threads, 0, stream>>>(t);
            else attention_kernel<T, D, false, true><<<grid, threads, 0, stream>>>(t);
        } else {
            attention_kernel<T, D, true, true><<<grid, threads, 0, stream>>>(t);
        }
    } else {
        const int64_t grid = ((pairs + 127) / 128 + t.S) * t.k_heads * t.parts;
        attention_kernel<T, D, true, false><<<dim3((unsigned)grid), dim3(256), 0, stream>>>(t);
    }
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && t.parts > 1) {
        attention_join_kernel<T><<<dim3((unsigned)((pairs * t.k_heads + 3) / 4)), dim3(256), 0, stream>>>(t);
        e = hipGetLastError();
    }
    return (int)e;
}

template <typename T>
int launch(const HopAttentionTask& t, const HopAttentionPlan& plan, hipStream_t stream) {
    launch_copies<T>(plan.copies, stream);
    auto fits = [&](const void* p, int64_t ld) { return ((uintptr_t)p & 15u) == 0 && (ld * sizeof(T)) % 16 == 0; };
    const bool fed = fits(t.q, t.ldq) && fits(t.k, t.ldk) && fits(t.v, t.ldv) && (t.head * sizeof(T)) % 16 == 0;
    return t.cols <= 64 ? launch<T, 64>(t, fed, stream) : launch<T, 128>(t, fed, stream);
}

int parts_of(const HopAttentionTask& t) {
    const int64_t step = few(t) ? 32 : 128, tiles = (((int64_t)t.q_rows * t.group + step - 1) / step + t.S) * t.k_heads, keys = t.k_rows / t.S;
    // Workgroups, and keys of a part: with few pairs a workgroup to a CU (the next token of 32 sequences of 2048 tokens, 32 heads on 8 of 128: 46.5 us, with two 54), and no parts where
    // its wavefronts have little to do (4000 keys in parts of 512 16 us, of 1024 20).
    const int64_t wanted = few(t) ? 256 : 512, least = few(t) ? 512 : 256;
    return (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>((wanted + tiles - 1) / tiles, keys / least), 64));
}

}  // namespace

HopAttentionPlan hopa_forward_plan(HopAttentionTask* task, int dtype, char* scratch) {
    HopAttentionTask& t = *task;
    HopAttentionPlan p = {};
    Planner planner(task, &p, dtype, scratch);
    const int heads = t.k_heads * t.group;
    t.parts = parts_of(t);
    if (t.parts > 1) t.partial = (float*)planner.take((size_t)t.parts * t.q_rows * heads * (t.cols + 2) * 4);
    const bool through_registers = t.cols <= 64 || (dtype == HOP_BF16 ? kThroughRegisters<bf16, 128> : kThroughRegisters<float, 128>);
    if (!few(t) || !through_registers) {
        planner.align(t.q, t.ldq, t.q_rows, heads, t.q_begin);
        planner.align(t.k, t.ldk, t.k_rows, t.k_heads, t.k_begin);
        planner.align(t.v, t.ldv, t.k_rows, t.k_heads, t.k_begin);
    }
    return p;
}

int hopa_forward(const HopAttentionTask& t, int dtype, const HopAttentionPlan& plan, void* stream) {
    return dtype == HOP_BF16 ? launch<bf16>(t, plan, (hipStream_t)stream) : launch<float>(t, plan, (hipStream_t)stream);
}
