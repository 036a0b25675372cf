// Gradients of softmax attention (hop_attention.hip), for gfx950 (CDNA4).
//
//   p_ij = exp(scale q_i k_j - lse_i),  D_i = sum_c do_ic o_ic,  ds_ij = p_ij (do_i v_j - D_i)
//   dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i,  dv_j = sum_i p_ij do_i              10 pairs cols operations
//
// Two kernels, each with sums of its own in registers, so that results are the same bits every time: one passes over the keys of a run of pairs for dq
// (and leaves D and lse for the other), one over the pairs of a run of keys for dk and dv.  The price is that scores and do v^T are computed
// twice: 14 operations where 10 would do.  Both take even shares of all tiles, which a small kernel in front of them lays out from the tables.
#include <algorithm>
#include <type_traits>

#include "hop_attention_device.h"

using namespace hopa;

namespace {

template <typename T, int D>
constexpr int kTileRows = D * (int)sizeof(T) <= 256 ? 64 : 32;
constexpr int kShift = 7, kTile = 1 << kShift;          // pairs or keys of a tile
// Workgroups on a CU at once: registers and LDS of one with 128 columns or fp32 leave no room for another.
template <typename T, int D>
constexpr int kBeside = sizeof(T) == 2 && D <= 64 ? 2 : 1;
constexpr int kCus = 256;

__device__ __forceinline__ int64_t pairs_of(const HopAttentionTask& t) { return (int64_t)t.q_rows * t.group; }
// The first pair that sees a key.
__device__ __forceinline__ int seen_from(const HopAttentionTask& t, int nq, int nk, int key) { return t.causal ? max(0, key - (nk - nq)) * t.group : 0; }

// ---- the plan -----------------------------------------------------------------------------
// A workgroup for the tiles of pairs, one for those of keys.  `rows`: of a stage.
constexpr int kPlanners = 1024;
__device__ __forceinline__ int64_t scan_all(int64_t v, int64_t* waves, int64_t* all) {          // sum of those in front
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t sum = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t before = __shfl_up(sum, o);
        if (lane >= o) sum += before;
    }
    __syncthreads();
    if (lane == 63) waves[wave] = sum;
    __syncthreads();
    int64_t front = 0, total = 0;
    for (int i = 0; i < kPlanners / 64; ++i) {
        if (i < wave) front += waves[i];
        total += waves[i];
    }
    *all = total;
    return front + sum - v;
}
__global__ __launch_bounds__(kPlanners) void attention_plan_kernel(HopAttentionTask t, int rows, int64_t most_q, int64_t most_k) {
    __shared__ int32_t first_tile[HOP_MAX_GROUPS + 1];
    __shared__ int64_t waves[kPlanners / 64];
    const bool of_keys = blockIdx.x == 1;
    const int64_t most = of_keys ? most_k : most_q;
    Plan* plan = (Plan*)(of_keys ? t.k_plan : t.q_plan);
    int64_t tiles = 0;
    for (int base = 0; base < t.S; base += kPlanners) {
        const int s = base + threadIdx.x;
        int b = 0, n = 0;
        if (s < t.S) rows_of(of_keys ? t.k_begin : t.q_begin, s, of_keys ? t.k_rows : t.q_rows, &b, &n);
        const int64_t its = ((int64_t)n * (of_keys ? 1 : t.group) + kTile - 1) >> kShift;
        int64_t all;
        const int64_t front = tiles + scan_all(its, waves, &all);
        if (s < t.S) first_tile[s] = (int32_t)(front < most ? front : most);          // beyond it only where a table is broken
        tiles += all;
    }
    if (tiles > most) tiles = most;
    __syncthreads();
    int64_t stages = 0;
    for (int64_t base = 0; base < tiles; base += kPlanners) {
        const int64_t at = base + threadIdx.x;
        int64_t n = 0;
        PlanTile tile = {};
        if (at < tiles) {
            int low = 0, high = t.S;                    // first_tile[low] <= at < first_tile[high]; of several with the same one the last has tiles
            while (high - low > 1) {
                const int middle = (low + high) / 2;
                if (first_tile[middle] <= at) low = middle;
                else high = middle;
            }
            rows_of(t.q_begin, low, t.q_rows, &tile.q0, &tile.nq);
            rows_of(t.k_begin, low, t.k_rows, &tile.k0, &tile.nk);
            tile.first = (int)(at - first_tile[low]) << kShift;
            const int pairs = tile.nq * t.group;
            if (of_keys) {
                n = (pairs - min(pairs, seen_from(t, tile.nq, tile.nk, tile.first) / rows * rows) + rows - 1) / rows;
            } else {
                const int last = divide(min(tile.first + kTile, pairs) - 1, t.group_inverse);
                n = ((t.causal ? clamp_int(last + 1 + tile.nk - tile.nq, 0, tile.nk) : tile.nk) + rows - 1) / rows;
            }
            if (n < 1) n = 1;                           // it has zeros to write
            tile.stages = (int32_t)n;
        }
        int64_t all;
        tile.before = stages + scan_all(n, waves, &all);
        if (at < tiles) plan->tile[at] = tile;
        stages += all;
    }
    if (threadIdx.x == 0) {
        PlanTile end = {};
        end.before = stages;
        plan->tile[tiles] = end;
        plan->stages = stages;
        plan->tiles = tiles;
    }
}

// Which run a workgroup takes: neighbours on the same XCD, whose second-level cache they share.
__device__ __forceinline__ int64_t run_of_block(int64_t blocks) {
    const int at = blockIdx.x, n = gridDim.x;
    return blocks == n && n % 8 == 0 ? (int64_t)(at % 8) * (n / 8) + at / 8 : at;
}
// A part's place: rows of `cols` floats.  A tile's first part is the last thing that its workgroup does, any other one the first, so there are two at most.
__device__ __forceinline__ float* part_place(const HopAttentionTask& t, int64_t block, bool first_part, int sums) {
    return t.partial + (block * 2 + (first_part ? 1 : 0)) * sums * kTile * t.cols;
}

// ---- dq ---------------------------------------------------------------------------------
template <typename T, int D, bool FED>
__global__ __launch_bounds__(256, (kBeside<T, D>)) void attention_dq_kernel(HopAttentionTask t) {
    typedef Tile<T, D> L;
    constexpr int NT = 256, kRows = kTileRows<T, D>, kBytes = kRows * L::kLine, kU = D / 32;
    constexpr int kStage = 2 * kBytes;                      // keys, values
    __shared__ __attribute__((aligned(16))) char pool[3 * kStage];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, hi = lane >> 5;
    const Runs runs(t.q_plan, t.k_heads, gridDim.x);
    const int64_t block = run_of_block(runs.blocks);
    if (block >= runs.blocks) return;
    const Place from = begin_of_run(runs, block), to = begin_of_run(runs, block + 1);

    for (int64_t number = from.tile; number < to.tile || (number == to.tile && to.stage > 0); ++number) {
        const int head = __builtin_amdgcn_readfirstlane((int)(number / runs.plan->tiles));
        const PlanTile seq = tile_of(runs, number - head * runs.plan->tiles);
        const int first_stage = __builtin_amdgcn_readfirstlane(number == from.tile ? from.stage : 0);
        const int last_stage = __builtin_amdgcn_readfirstlane(number == to.tile ? to.stage : seq.stages);
        const Sequence its_rows = {seq.q0, seq.nq, seq.k0, seq.nk};
        const int pairs = seq.nq * t.group, first = seq.first, mine = first + wave * 32, pair = mine + (lane & 31);
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
        if (live && !hi && first_stage == 0) {
            HOPL_GLOBAL float* terms = (HOPL_GLOBAL float*)t.terms + head * pairs_of(t) + (int64_t)seq.q0 * t.group + pair;
            terms[0] = lse;
            terms[t.k_heads * pairs_of(t)] = delta;
        }
        const int limit = live ? visible(its_rows, t.causal, row) : seq.nk;
        auto visible_of = [&](int p) { return visible(its_rows, t.causal, divide(p, t.group_inverse)); };
        const int all_see = visible_of(min(mine, pairs - 1)), all_see_here = visible_of(first);
        const int end = min(visible_of(min(first + kTile, pairs) - 1), last_stage * kRows), begin = first_stage * kRows;

        const Rows gk = {t.ldk, 1, 0, t.cols}, gv = {t.ldv, 1, 0, t.cols};
        Feed<T, D, kRows, NT, FED, false> feed_k, feed_v;
        feed_k.begin(gk, 0);
        feed_v.begin(gv, 0);
        auto issue = [&](char* b, int i) __attribute__((always_inline)) {
            const int key = begin + i * kRows;
            feed_k.issue(b, k, gk, key, seq.nk - key);
            feed_v.issue(b + kBytes, v, gv, key, seq.nk - key);
        };
        auto put = [&](char* b) __attribute__((always_inline)) {
            feed_k.put(b);
            feed_v.put(b + kBytes);
        };
        f32x16 dq[kU], p, ds;
        // the scores of the unit at `next` (or none), beside a unit's own gradients of scores and what they add
        auto step = [&](const char* b, int key, const char* next) __attribute__((always_inline)) {
            f32x16 next_p, next_ds;
            scores_beside<T, D, true>(next, next + kBytes, fq, fg, next_p, next_ds,
                                      [&](int r) __attribute__((always_inline)) { ds[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[r], t.scale_log2, -lse)) * (ds[r] - delta); });
            Sums<T, D, false> sums;
            sums.begin(b, b);
            if (key + 32 > all_see) {
                asm volatile("");              // a branch, which few tiles take, and not selections that all of them make
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (key + 8 * (r >> 2) + 4 * hi + (r & 3) >= limit) ds[r] = 0.f;
            }
            const Weights<T> w(ds);
            sums.add(b, b, w, w, dq, dq);
            p = next_p;
            ds = next_ds;
        };
        auto scores = [&](const char* b) __attribute__((always_inline)) { scores_beside<T, D, true>(b, b + kBytes, fq, fg, p, ds, [](int) {}); };
        auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int c = 0; c < kU; ++c) dq[c] = (f32x16)(0.f);
        };
        clear();
        if (begin < end)
            pipeline<kRows / 32>((end - begin + kRows - 1) / kRows, pool, kStage, issue, put, scores, [&](int i, const char* b, int u, const char* next, int next_u) __attribute__((always_inline)) {
                step(b + 32 * u * L::kLine, begin + i * kRows + 32 * u, next + 32 * next_u * L::kLine);
            });
        if (t.causal && __syncthreads_or(live && !all_finite(dq))) {
            clear();
            for (int key = begin; key < end; key += kRows) {
                __syncthreads();
                issue(pool, (key - begin) / kRows);
                put(pool);
                arrive();
                if (key + kRows > all_see_here) {
                    add_not_finite<T, D>(pool, min(kRows, seq.nk - key), dq, [&](int j) { return key + j < limit; });
                    __syncthreads();
                    drop_not_finite<T, kBytes, NT>(pool);
                    __syncthreads();
                }
                for (int u = 0; u < kRows / 32; ++u) {
                    scores(pool + 32 * u * L::kLine);
                    step(pool + 32 * u * L::kLine, key + 32 * u, pool);
                }
            }
        }
        if (!live) continue;
        if (first_stage > 0 || last_stage < seq.stages)
            store_columns<float, D>(part_place(t, block, first_stage == 0, 1) + (int64_t)(pair - first) * t.cols, t.cols, dq, 1.f);
        else
            store_columns<T, D>((T*)t.dq + at * t.lddq + column, t.cols, dq, t.scale);
    }
}

// ---- dk and dv ------------------------------------------------------------------------------
template <typename T, int D, bool FED>
__global__ __launch_bounds__(256, (kBeside<T, D>)) void attention_dkv_kernel(HopAttentionTask t) {
    typedef Tile<T, D> L;
    constexpr int NT = 256, kRows = kTileRows<T, D>, kBytes = kRows * L::kLine, kU = D / 32;
    constexpr int kStage = 2 * kBytes + 512;                // queries, gradients, lse log2(e) of 64 pairs, their D
    __shared__ __attribute__((aligned(16))) char pool[3 * kStage];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, hi = lane >> 5;
    const Runs runs(t.k_plan, t.k_heads, gridDim.x);
    const int64_t block = run_of_block(runs.blocks);
    if (block >= runs.blocks) return;
    const Place from = begin_of_run(runs, block), to = begin_of_run(runs, block + 1);

    for (int64_t number = from.tile; number < to.tile || (number == to.tile && to.stage > 0); ++number) {
        const int head = __builtin_amdgcn_readfirstlane((int)(number / runs.plan->tiles));
        const PlanTile seq = tile_of(runs, number - head * runs.plan->tiles);
        const int first_stage = __builtin_amdgcn_readfirstlane(number == from.tile ? from.stage : 0);
        const int last_stage = __builtin_amdgcn_readfirstlane(number == to.tile ? to.stage : seq.stages);
        const int first = seq.first, mine = first + wave * 32, key = mine + (lane & 31);
        const bool live = key < seq.nk;
        const int64_t at = seq.k0 + (live ? key : 0);
        const int pairs = seq.nq * t.group;
        const T* q = (const T*)t.q + seq.q0 * t.ldq + head * t.group * t.cols;
        const T* g = (const T*)t.grad + seq.q0 * t.ldgrad + head * t.group * t.cols;
        const float* terms = t.terms + head * pairs_of(t) + (int64_t)seq.q0 * t.group;

        typename L::frag fk[L::kSteps], fv[L::kSteps];
        load_columns<T, D, FED>(fk, (const T*)t.k + at * t.ldk + head * t.cols, t.cols, live);
        load_columns<T, D, FED>(fv, (const T*)t.v + at * t.ldv + head * t.cols, t.cols, live);
        const int least = live ? seen_from(t, seq.nq, seq.nk, key) : 0;
        const int all_see = seen_from(t, seq.nq, seq.nk, min(mine + 32, seq.nk) - 1), all_see_here = seen_from(t, seq.nq, seq.nk, min(first + kTile, seq.nk) - 1);
        const int start = min(pairs, seen_from(t, seq.nq, seq.nk, first) / kRows * kRows);
        const int begin = start + first_stage * kRows, end = min(pairs, start + last_stage * kRows);
        const Rows gq = {t.ldq, t.group, t.group_inverse, t.cols}, gg = {t.ldgrad, t.group, t.group_inverse, t.cols};
        Feed<T, D, kRows, NT, FED, true> feed_q, feed_g;
        feed_q.begin(gq, 0);
        feed_g.begin(gg, 0);
        auto issue = [&](char* b, int i) __attribute__((always_inline)) {
            const int pair = begin + i * kRows;
            feed_q.issue(b, q, gq, pair, pairs - pair);
            feed_g.issue(b + kBytes, g, gg, pair, pairs - pair);
            if (wave < 2) {
                const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)(terms + wave * t.k_heads * pairs_of(t) + pair), 0,
                                                                                   min(kRows, pairs - pair) * 4, 0x00020000);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(b + 2 * kBytes + wave * 256), 4, lane * 4, 0, 0, 0);
            }
        };
        auto put = [&](char* b) __attribute__((always_inline)) {
            feed_q.put(b);
            feed_g.put(b + kBytes);
        };
        f32x16 dk[kU], dv[kU], p, ds;
        auto step = [&](const char* b, const char* terms_of_unit, int pair, const char* next) __attribute__((always_inline)) {
            f32x16 next_p, next_ds;
            f32x4 lse[4], delta[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                lse[i] = *(const f32x4*)(terms_of_unit + 32 * i + 16 * hi);
                delta[i] = *(const f32x4*)(terms_of_unit + 256 + 32 * i + 16 * hi);
            }
            scores_beside<T, D, true>(next, next + kBytes, fk, fv, next_p, next_ds, [&](int r) __attribute__((always_inline)) {
                p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[r], t.scale_log2, -lse[r >> 2][r & 3]));
                ds[r] = p[r] * (ds[r] - delta[r >> 2][r & 3]);
            });
            Sums<T, D, true> sums;
            sums.begin(b + kBytes, b);
            if (pair < all_see) {
                asm volatile("");              // a branch, as above
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (pair + 8 * (r >> 2) + 4 * hi + (r & 3) < least) p[r] = ds[r] = 0.f;
            }
            const Weights<T> wp(p), ws(ds);
            sums.add(b + kBytes, b, wp, ws, dv, dk);
            p = next_p;
            ds = next_ds;
        };
        auto scores = [&](const char* b) __attribute__((always_inline)) { scores_beside<T, D, true>(b, b + kBytes, fk, fv, p, ds, [](int) {}); };
        auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int c = 0; c < kU; ++c) dk[c] = dv[c] = (f32x16)(0.f);
        };
        clear();
        if (begin < end)
            pipeline<kRows / 32>((end - begin + kRows - 1) / kRows, pool, kStage, issue, put, scores, [&](int i, const char* b, int u, const char* next, int next_u) __attribute__((always_inline)) {
                step(b + 32 * u * L::kLine, b + 2 * kBytes + 128 * u, begin + i * kRows + 32 * u, next + 32 * next_u * L::kLine);
            });
        if (t.causal && __syncthreads_or(live && !(all_finite(dk) && all_finite(dv)))) {
            clear();
            for (int pair = begin; pair < end; pair += kRows) {
                __syncthreads();
                issue(pool, (pair - begin) / kRows);
                put(pool);
                arrive();
                if (pair < all_see_here) {
                    const int count = min(kRows, pairs - pair);
                    add_not_finite<T, D>(pool, count, dk, [&](int j) { return pair + j >= least; });
                    add_not_finite<T, D>(pool + kBytes, count, dv, [&](int j) { return pair + j >= least; });
                    __syncthreads();
                    drop_not_finite<T, kBytes, NT>(pool);
                    drop_not_finite<T, kBytes, NT>(pool + kBytes);
                    __syncthreads();
                }
                for (int u = 0; u < kRows / 32; ++u) {
                    scores(pool + 32 * u * L::kLine);
                    step(pool + 32 * u * L::kLine, pool + 2 * kBytes + 128 * u, pair + 32 * u, pool);
                }
            }
        }
        if (!live) continue;
        if (first_stage > 0 || last_stage < seq.stages) {
            float* part = part_place(t, block, first_stage == 0, 2) + (int64_t)(key - first) * t.cols;
            store_columns<float, D>(part, t.cols, dk, 1.f);
            store_columns<float, D>(part + kTile * t.cols, t.cols, dv, 1.f);
        } else {
            store_columns<T, D>((T*)t.dk + at * t.lddk + head * t.cols, t.cols, dk, t.scale);
            store_columns<T, D>((T*)t.dv + at * t.lddv + head * t.cols, t.cols, dv, 1.f);
        }
    }
}

// ---- parts, joined in their order: 16 rows of a tile ------------------------------------------
// `sums` matrices to a part: dq, or dk and dv.
template <typename T, bool KEYS>
__global__ __launch_bounds__(256) void attention_grad_join_kernel(HopAttentionTask t, int most) {
    const Runs runs(KEYS ? t.k_plan : t.q_plan, t.k_heads, most);
    const int64_t tiles = runs.plan->tiles;
    constexpr int kSums = KEYS ? 2 : 1, kEach = kTile / 16;
    const int64_t number = blockIdx.x / kEach;
    if (number >= tiles * t.k_heads) return;
    const int head = (int)(number / tiles), first = blockIdx.x % kEach * 16;
    const PlanTile seq = tile_of(runs, number - head * tiles);
    int64_t b0, b1;
    if (!runs_inside(runs, head, seq, &b0, &b1)) return;
    const int all = (KEYS ? seq.nk : seq.nq * t.group) - seq.first, rows = min(16, all - first);
    for (int i = threadIdx.x; i < rows * t.cols; i += 256) {
        const int r = i / t.cols, c = i - r * t.cols, in = first + r, n = seq.first + in;
        const int64_t place = (int64_t)in * t.cols + c;
#pragma unroll
        for (int which = 0; which < kSums; ++which) {
            float v = ((const HOPL_GLOBAL float*)part_place(t, b0 - 1, true, kSums))[which * kTile * t.cols + place];
            for (int64_t b = b0; b <= b1; ++b) v += ((const HOPL_GLOBAL float*)part_place(t, b, false, kSums))[which * kTile * t.cols + place];
            if constexpr (KEYS) {
                const int64_t at = seq.k0 + n;
                if (which) ((HOPL_GLOBAL T*)t.dv)[at * t.lddv + head * t.cols + c] = (T)v;
                else ((HOPL_GLOBAL T*)t.dk)[at * t.lddk + head * t.cols + c] = (T)(v * t.scale);
            } else {
                const int row = divide(n, t.group_inverse);
                ((HOPL_GLOBAL T*)t.dq)[(int64_t)(seq.q0 + row) * t.lddq + (head * t.group + n - row * t.group) * t.cols + c] = (T)(v * t.scale);
            }
        }
    }
}

template <typename T, int D, bool FED>
int launch(const HopAttentionTask& t, const HopAttentionPlan& plan, hipStream_t stream) {
    const int grid = kCus * kBeside<T, D>;
    constexpr int kJoins = kTile / 16;
    attention_plan_kernel<<<dim3(2), dim3(kPlanners), 0, stream>>>(t, kTileRows<T, D>, plan.q_tiles, plan.k_tiles);
    if (t.q_rows) {
        attention_dq_kernel<T, D, FED><<<dim3(grid), dim3(256), 0, stream>>>(t);
        (attention_grad_join_kernel<T, false>)<<<dim3((unsigned)(plan.q_tiles * t.k_heads * kJoins)), dim3(256), 0, stream>>>(t, grid);
    }
    if (t.k_rows) {
        attention_dkv_kernel<T, D, FED><<<dim3(grid), dim3(256), 0, stream>>>(t);
        (attention_grad_join_kernel<T, true>)<<<dim3((unsigned)(plan.k_tiles * t.k_heads * kJoins)), dim3(256), 0, stream>>>(t, grid);
    }
    return (int)hipGetLastError();
}

template <typename T>
int launch(const HopAttentionTask& t, const HopAttentionPlan& plan, hipStream_t stream) {
    auto fits = [&](const void* p, int64_t ld) { return ((uintptr_t)p & 15u) == 0 && (ld * sizeof(T)) % 16 == 0; };
    const bool fed = fits(t.q, t.ldq) && fits(t.k, t.ldk) && fits(t.v, t.ldv) && fits(t.grad, t.ldgrad) && fits(t.o, t.ldo) && (t.cols * sizeof(T)) % 16 == 0;
    if (t.cols <= 64) return fed ? launch<T, 64, true>(t, plan, stream) : launch<T, 64, false>(t, plan, stream);
    return fed ? launch<T, 128, true>(t, plan, stream) : launch<T, 128, false>(t, plan, stream);
}

}  // namespace

HopAttentionPlan hopa_grad_plan(const HopAttentionTask& t, int dtype) {
    HopAttentionPlan p;
    p.q_tiles = ((int64_t)t.q_rows * t.group + kTile - 1) / kTile + t.S;
    p.k_tiles = ((int64_t)t.k_rows + kTile - 1) / kTile + t.S;
    auto bytes = [](int64_t tiles) { return (size_t)((sizeof(Plan) + tiles * sizeof(PlanTile) + 255) / 256 * 256); };
    p.q_bytes = bytes(p.q_tiles);
    p.k_bytes = bytes(p.k_tiles);
    // two parts of a workgroup, dk and dv at most; fewer tiles than workgroups are cut only into as many
    const int blocks = kCus * (dtype == HOP_BF16 && t.cols <= 64 ? 2 : 1);
    p.partial_bytes = (size_t)blocks * 2 * 2 * kTile * t.cols * 4;
    return p;
}

int hopa_grad(const HopAttentionTask& t, int dtype, const HopAttentionPlan& plan, void* stream) {
    return dtype == HOP_BF16 ? launch<bf16>(t, plan, (hipStream_t)stream) : launch<float>(t, plan, (hipStream_t)stream);
}
