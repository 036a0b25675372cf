// Gradients of softmax attention (hop_attention.hip), for gfx950 (CDNA4).
//
//   p_ij = exp(scale q_i k_j - lse_i),  D_i = sum_c do_ic o_ic,  ds_ij = p_ij (do_i v_j - D_i)
//   dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i,  dv_j = sum_i p_ij do_i              10 pairs cols operations
//
// Two kernels, each with sums of its own in registers, so that results are the same bits every time: one passes over the keys of a tile of pairs for dq
// (and leaves D and lse for the other), one over the pairs of a tile of keys for dk and dv.  The price is that scores and do v^T are computed
// twice: 14 operations where 10 would do.  Both take even shares of all tiles, which a small kernel in front of them lays out from the tables: with a workgroup to a tile
// the longest sequence's tiles decided (12288 tokens in 6 sequences, 16 heads on 2: 1076 us, now 458).
//
// What bounds them is the matrix unit, at the clock that its power leaves: 8192 tokens that all see each other, 16 heads of 128 columns on 2, bfloat16, take 1716 us,
// 1120 TFLOP/s of the 14 operations (a large library product reaches 1230 to 1390 on such numbers); 58 % of the cycles have a product under way.
#include <algorithm>
#include <type_traits>

#include "hop_attention_device.h"

using namespace hopa;

namespace {

constexpr int kShift = 7, kTile = 1 << kShift;          // pairs or keys of a tile, 32 of a wavefront
static_assert(kTile <= kHopaMostTileRows, "their distance");
constexpr int kCus = 256;
// kSkip: units that a wavefront's columns see nothing of are left out in fp32, whose products take long (32 sequences of 128 rows: 99 us, with them 103); in bfloat16 the other
// wavefronts of the stage decide and the branch costs more than it saves (8192 rows, causal: 1003 us, without it 960).
template <typename T>
constexpr bool kSkip = sizeof(T) == 4;
constexpr int kExact = 128;                             // keys: see attention_dq_kernel
// Two halves of a workgroup with the same tile take every other 32 rows of a stage, so that a SIMD has two wavefronts, of which one computes while the other waits, and the CU
// only one set of tiles (one wavefront with twice the registers issues an instruction every 5 cycles at best, which is too few beside its products: 1860 us for the above).  In fp32 with 128 columns the sums and operands of one wavefront fill a SIMD's registers.
template <typename T, int D>
constexpr int kHalves = D * (int)sizeof(T) <= 256 ? 2 : 1;

__device__ __forceinline__ int64_t pairs_of(const HopAttentionTask& t) { return (int64_t)t.q_rows * t.group; }
// The first pair that sees a key.
__device__ __forceinline__ int seen_from(const HopAttentionTask& t, int nq, int nk, int key) { return t.causal ? max(0, key - (nk - nq)) * t.group : 0; }

// ---- the plan -----------------------------------------------------------------------------
// A workgroup for the tiles of pairs, one for those of keys.  `rows`: of a stage.
constexpr int kPlanners = 1024;
// What a tile takes beside its stages, in stages: 17500 cycles for pairs, of which a stage of 128 columns in bfloat16 takes 2440, and more for keys.  12288 tokens, 16 heads on 2:
// dq and dk, dv in 215 and 237 us; as if a tile took nothing 439 and 272.  Measured there; fewer columns and fp32 have stages of
// other lengths and are weighed by the same numbers.
constexpr int kPairsFixed = 8, kKeysFixed = 10;
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
    const int fixed = of_keys ? kKeysFixed : kPairsFixed;
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
    int64_t weight = 0;
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
                const int last = hopa_divide(min(tile.first + kTile, pairs) - 1, t.group_inverse, t.group_shift);
                n = ((t.causal ? clamp_int(last + 1 + tile.nk - tile.nq, 0, tile.nk) : tile.nk) + rows - 1) / rows;
            }
            if (n < 1) n = 1;                           // it has zeros to write
            tile.stages = (int32_t)n;
        }
        int64_t all;
        tile.before = weight + scan_all(at < tiles ? n + fixed : 0, waves, &all);
        if (at < tiles) plan->tile[at] = tile;
        weight += all;
    }
    if (threadIdx.x == 0) {
        PlanTile end = {};
        end.before = weight;
        plan->tile[tiles] = end;
        plan->weight = weight;
        plan->tiles = tiles;
        plan->fixed = fixed;
    }
}

// Which run a workgroup takes: neighbours on the same XCD, whose second-level cache they share.
__device__ __forceinline__ int64_t run_of_block(int64_t blocks) {
    const int at = blockIdx.x, n = gridDim.x;
    return blocks == n && n % 8 == 0 ? (int64_t)(at % 8) * (n / 8) + at / 8 : at;
}
// A part's place: rows of `cols` floats.  A tile's first part is the last thing that its workgroup does, any other one the first, so there are two at most.
// Those of dq, one matrix each, lie in front of those of dk and dv, two each.
template <bool KEYS>
__device__ __forceinline__ float* part_place(const HopAttentionTask& t, int64_t block, bool first_part) {
    const int64_t matrix = kTile * t.cols, number = block * 2 + (first_part ? 1 : 0);
    return t.partial + (KEYS ? kCus * 2 + number * 2 : number) * matrix;
}

// The second half's sums, added to the first one's.  Nobody uses the pool any more.
template <int N, int HALVES>
__device__ __forceinline__ void add_halves(char* pool, int half, int wave, f32x16 (&sum)[N]) {
    if constexpr (HALVES == 2) {
        char* mine = pool + (wave * N * 4 * 64 + (threadIdx.x & 63)) * 16;
        if (half)
#pragma unroll
            for (int c = 0; c < N; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) *(f32x4*)(mine + (c * 4 + e) * 1024) = {sum[c][4 * e], sum[c][4 * e + 1], sum[c][4 * e + 2], sum[c][4 * e + 3]};
        __syncthreads();
        if (!half)
#pragma unroll
            for (int c = 0; c < N; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const f32x4 more = *(const f32x4*)(mine + (c * 4 + e) * 1024);
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum[c][4 * e + i] += more[i];
                }
    }
}

// ---- dq ---------------------------------------------------------------------------------
template <typename T, int D>
__global__ __launch_bounds__((256 * kHalves<T, D>), (kHalves<T, D>)) void attention_dq_kernel(HopAttentionTask t) {
    typedef Tile<T, D> L;
    typedef Weights<T> W;
    constexpr int kH = kHalves<T, D>, NT = 256 * kH, kRows = 32 * kH, kBytes = kRows * L::kLine, kU = D / 32, kS = L::kSteps;
    constexpr int kStage = 2 * kBytes;                      // keys, values
    __shared__ __attribute__((aligned(16))) char pool[2 * kStage];
    __shared__ int not_finite;
    __shared__ float exact[2][kTile];
    const int half = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6 & 3), lane = threadIdx.x & 63, hi = lane >> 5;
    const Places<T, D> all_places;
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
        const int row = live ? hopa_divide(pair, t.group_inverse, t.group_shift) : 0, its = live ? pair - row * t.group : 0;
        const int64_t at = seq.q0 + row;
        const int column = (head * t.group + its) * t.cols;
        const T* k = (const T*)t.k + seq.k0 * t.ldk + head * t.head;
        const T* v = (const T*)t.v + seq.k0 * t.ldv + head * t.head;

        const int limit = live ? visible(its_rows, t.causal, row) : seq.nk;
        auto visible_of = [&](int p) { return visible(its_rows, t.causal, hopa_divide(p, t.group_inverse, t.group_shift)); };
        const int all_see = visible_of(min(mine, pairs - 1)), all_see_here = visible_of(first), some_see = mine < pairs ? visible_of(min(mine + 32, pairs) - 1) : 0;
        const int end = min(visible_of(min(first + kTile, pairs) - 1), last_stage * kRows), begin = first_stage * kRows;

        const Rows gk = {t.ldk, 1, 0, 0, t.head}, gv = {t.ldv, 1, 0, 0, t.head};
        Feed<T, D, kRows, NT, true, false> feed_k, feed_v;
        feed_k.begin(gk, 0);
        feed_v.begin(gv, 0);
        auto issue = [&](char* b, int i) __attribute__((always_inline)) {
            const int key = begin + i * kRows;
            feed_k.issue(b, k, gk, key, seq.nk - key);
            feed_v.issue(b + kBytes, v, gv, key, seq.nk - key);
        };
        const int n = begin < end ? (end - begin + kRows - 1) / kRows : 0;
        // The tile's queries, gradients and results come through the buffers of the stages.
        const Rows gq = {t.ldq, t.group, t.group_inverse, t.group_shift, t.head}, gg = {t.ldgrad, t.group, t.group_inverse, t.group_shift, t.head}, go = {t.ldo, t.group, t.group_inverse, t.group_shift, t.head};
        Feed<T, D, kTile, NT, true, true> feed;
        typename L::frag fq[kS], fg[kS];
        char* const second = kH == 2 ? pool + kStage : pool;
        const int in_tile = 32 * wave * L::kLine;
        auto fetch_tile = [&](char* to, const void* m, const Rows& g) __attribute__((always_inline)) {
            feed.begin(g, first - hopa_divide(first, t.group_inverse, t.group_shift) * t.group);
            feed.issue(to, (const T*)m + seq.q0 * g.ld + head * t.group * t.head, g, first, pairs - first);
        };
        __syncthreads();                                   // with whoever still reads from the buffers
        if (threadIdx.x == 0) not_finite = 0;
        fetch_tile(pool, t.q, gq);
        if (kH == 2) fetch_tile(second, t.grad, gg);
        arrive();
        take_columns<T, D>(fq, pool + in_tile, all_places.along);
        if (kH == 1) {
            arrive();
            fetch_tile(second, t.grad, gg);
            arrive();
        }
        take_columns<T, D>(fg, second + in_tile, all_places.along);
        arrive();
        fetch_tile(second, t.o, go);
        if (kH == 2 && n) issue(pool, 0);
        const float lse = live ? ((const HOPL_GLOBAL float*)t.lse)[(int64_t)(head * t.group + its) * t.q_rows + at] * (1.f / kLn2) : 0.f;
        arrive();
        float delta = 0.f;
#pragma unroll
        for (int i = 0; i < kS; ++i) {
            const typename L::frag fo = L::along(second + in_tile, all_places.along, i);
#pragma unroll
            for (int e = 0; e < L::kChunk; ++e) delta = __builtin_fmaf((float)fo[e], (float)fg[i][e], delta);
        }
        if (kH == 1) {
            arrive();
            if (n) issue(pool, 0);
        }
        delta = both_sum(delta);
        // With few keys to a query o's rounding weighs: D once more, as sum_j p_ij do_i v_j, which is exact to fp32's rounding and costs these tiles two products more.
        if (sizeof(T) == 2 && n && seq.stages * kRows <= kExact) {
            float sum = 0.f;
            stages(n, pool, kStage, issue, [&](const char* b, int i) __attribute__((always_inline)) {
                const int key = i * kRows + 32 * half;
                const char* sk = b + 32 * half * L::kLine;
                f32x16 p = (f32x16)(0.f), g = (f32x16)(0.f);
#pragma unroll
                for (int j = 0; j < kS; ++j) {
                    p = multiply(L::along(sk, all_places.along, j), fq[j], p);
                    g = multiply(L::along(sk + kBytes, all_places.along, j), fg[j], g);
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float term = __builtin_amdgcn_exp2f(__builtin_fmaf(p[r], t.scale_log2, -lse)) * g[r];
                    sum += key + 8 * (r >> 2) + 4 * hi + (r & 3) < limit ? term : 0.f;
                }
            });
            sum = both_sum(sum);
            exact[half][wave * 32 + (lane & 31)] = sum;
            __syncthreads();
            delta = exact[0][wave * 32 + (lane & 31)] + exact[1][wave * 32 + (lane & 31)];
            issue(pool, 0);
        }
        if (live && !hi && !half && first_stage == 0) {
            HOPL_GLOBAL float* terms = (HOPL_GLOBAL float*)t.terms + head * pairs_of(t) + (int64_t)seq.q0 * t.group + pair;
            terms[0] = lse;
            terms[t.k_heads * pairs_of(t)] = delta;
        }
        f32x16 dq[kU];
        // Scores; do v^T beside their exponentials; sums of the first 16 keys beside the second 16's gradients, then of those.
        auto work = [&](const char* b, int i) __attribute__((always_inline)) {
            const Places<T, D> places = all_places.again();
            const int key = begin + i * kRows + 32 * half;
            if (kSkip<T> && key >= some_see) return;                      // all of it is hidden from the wavefront's pairs
            const char* sk = b + 32 * half * L::kLine;
            const char* sv = sk + kBytes;
            constexpr int kN = 2 * kS + 2 * kU, kAhead = sizeof(T) == 4 ? 2 : 4, kFrom = kS + (sizeof(T) == 4 ? 1 : 2);
            typename L::frag a[kAhead];
            typename W::Part c[kAhead];
            auto fetch = [&](auto n) __attribute__((always_inline)) {
                constexpr int j = decltype(n)::value;
                if constexpr (j < kS) a[j % kAhead] = L::along(sk, places.along, j);
                else if constexpr (j < 2 * kS) a[j % kAhead] = L::along(sv, places.along, j - kS);
                else if constexpr (j < kN) c[j % kAhead] = W::template across<D>(sk, places.across, (j - 2 * kS) % kU, (j - 2 * kS) / kU);
            };
            f32x16 p = (f32x16)(0.f), ds = (f32x16)(0.f);
            static_for<kAhead>([&](auto n) __attribute__((always_inline)) { fetch(n); });
            static_for<2 * kS>([&](auto n) __attribute__((always_inline)) {
                constexpr int j = decltype(n)::value;
                __builtin_amdgcn_sched_barrier(0);
                if constexpr (j < kS) p = multiply(a[j % kAhead], fq[j], p);
                else ds = multiply(a[j % kAhead], fg[j - kS], ds);
                fetch(std::integral_constant<int, j + kAhead>());
                if constexpr (j >= kFrom)
#pragma unroll
                    for (int r = (j - kFrom) * 16 / (2 * kS - kFrom); r < (j - kFrom + 1) * 16 / (2 * kS - kFrom); ++r)
                        p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[r], t.scale_log2, -lse));
            });
            __builtin_amdgcn_sched_barrier(0);
            float less = delta;
            if (key + 32 > all_see) {
                asm volatile("");              // a branch, which few tiles take, and not selections that all of them make
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    ds[r] = key + 8 * (r >> 2) + 4 * hi + (r & 3) < limit ? p[r] * (ds[r] - delta) : 0.f;
                    p[r] = 1.f;
                }
                less = 0.f;
            }
#pragma unroll
            for (int r = 0; r < 8; ++r) ds[r] = p[r] * (ds[r] - less);
            static_for<2 * kU>([&](auto n) __attribute__((always_inline)) {
                constexpr int j = decltype(n)::value;
                dq[j % kU] = W::add(c[(j + 2 * kS) % kAhead], W::part_of(ds, j / kU), dq[j % kU]);
                fetch(std::integral_constant<int, j + 2 * kS + kAhead>());
                if constexpr (j < kU)
#pragma unroll
                    for (int r = 8 + j * 8 / kU; r < 8 + (j + 1) * 8 / kU; ++r) ds[r] = p[r] * (ds[r] - less);
                __builtin_amdgcn_sched_barrier(0);
            });
        };
        auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int c = 0; c < kU; ++c) dq[c] = (f32x16)(0.f);
        };
        clear();
        if (n) stages(n, pool, kStage, issue, work);
        if (!n) __syncthreads();                           // the stages have theirs
        if (t.causal && live && !all_finite(dq)) not_finite = 1;
        __syncthreads();
        if (not_finite) {
            clear();
            for (int i = 0; i < n; ++i) {
                const int key = begin + i * kRows;
                __syncthreads();
                issue(pool, i);
                arrive();
                if (key + kRows > all_see_here) {
                    add_not_finite<T, D, D>(pool, 0, 32 * half, min(32 * half + 32, seq.nk - key), dq, [&](int j) { return key + j < limit; });
                    __syncthreads();
                    drop_not_finite<T, kBytes, NT>(pool);
                    __syncthreads();
                }
                work(pool, i);
            }
            __syncthreads();
        }
        add_halves<kU, kH>(pool, half, wave, dq);
        if (!live || half) continue;
        if (first_stage > 0 || last_stage < seq.stages)
            store_columns<float, D>(part_place<false>(t, block, first_stage == 0) + (int64_t)(pair - first) * t.cols, t.cols, dq, 1.f);
        else
            store_columns<T, D>((T*)t.dq + at * t.lddq + column, t.cols, dq, t.scale);
    }
}

// ---- dk and dv ------------------------------------------------------------------------------
template <typename T, int D>
__global__ __launch_bounds__((256 * kHalves<T, D>), (kHalves<T, D>)) void attention_dkv_kernel(HopAttentionTask t) {
    typedef Tile<T, D> L;
    typedef Weights<T> W;
    constexpr int kH = kHalves<T, D>, NT = 256 * kH, kRows = 32 * kH, kBytes = kRows * L::kLine, kS = L::kSteps;
    constexpr int kStage = 2 * kBytes + 512;                // queries, gradients, lse log2(e) of the pairs, their D
    // Both sums of 128 columns leave no registers for the keys and values: there they wait in LDS.
    constexpr bool kHeld = kH == 1 || D * sizeof(T) <= 128;
    // In fp32 keys, values and both sums of 128 columns are more than all registers of a SIMD: the sums are made 64 columns at a time, each from scores of its own.
    constexpr int kCuts = kH == 1 ? 2 : 1, kSumCols = D / kCuts, kU = kSumCols / 32;
    __shared__ __attribute__((aligned(16))) char pool[2 * kStage], tile[kHeld ? 16 : 2 * kTile * L::kLine], zeros[128];
    __shared__ int not_finite;
    const int half = __builtin_amdgcn_readfirstlane(threadIdx.x >> 8), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6 & 3), lane = threadIdx.x & 63, hi = lane >> 5;
    if (threadIdx.x < 32) ((float*)zeros)[threadIdx.x] = 0.f;
    const Places<T, D> all_places;
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
        const T* q = (const T*)t.q + seq.q0 * t.ldq + head * t.group * t.head;
        const T* g = (const T*)t.grad + seq.q0 * t.ldgrad + head * t.group * t.head;
        const float* terms = t.terms + head * pairs_of(t) + (int64_t)seq.q0 * t.group;

        const int least = live ? seen_from(t, seq.nq, seq.nk, key) : 0;
        const int some_see = mine < seq.nk ? seen_from(t, seq.nq, seq.nk, mine) : pairs;
        const int all_see = seen_from(t, seq.nq, seq.nk, min(mine + 32, seq.nk) - 1), all_see_here = seen_from(t, seq.nq, seq.nk, min(first + kTile, seq.nk) - 1);
        const int start = min(pairs, seen_from(t, seq.nq, seq.nk, first) / kRows * kRows);
        const int begin = start + first_stage * kRows, end = min(pairs, start + last_stage * kRows);
        const Rows gq = {t.ldq, t.group, t.group_inverse, t.group_shift, t.head}, gg = {t.ldgrad, t.group, t.group_inverse, t.group_shift, t.head};
        Feed<T, D, kRows, NT, true, true> feed_q, feed_g;
        feed_q.begin(gq, 0);
        feed_g.begin(gg, 0);
        auto issue = [&](char* b, int i) __attribute__((always_inline)) {
            const int pair = begin + i * kRows;
            feed_q.issue(b, q, gq, pair, pairs - pair);
            feed_g.issue(b + kBytes, g, gg, pair, pairs - pair);
            if (!half && wave < 2) {
                const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void*)(terms + wave * t.k_heads * pairs_of(t) + pair), 0,
                                                                                   min(kRows, pairs - pair) * 4, 0x00020000);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(b + 2 * kBytes + wave * 256), 4, lane * 4, 0, 0, 0);
            }
        };
        const int n = begin < end ? (end - begin + kRows - 1) / kRows : 0;
        const Rows gk = {t.ldk, 1, 0, 0, t.head}, gv = {t.ldv, 1, 0, 0, t.head};
        Feed<T, D, kTile, NT, true, false> feed;
        auto fetch_tile = [&](char* to, const void* m, const Rows& g) __attribute__((always_inline)) {
            feed.begin(g, 0);
            feed.issue(to, (const T*)m + seq.k0 * g.ld + head * t.head, g, first, seq.nk - first);
        };
        const int in_tile = 32 * wave * L::kLine;
        const char *const keys = tile + in_tile, *const values = keys + kTile * L::kLine;
        typename L::frag fk[kHeld ? kS : 1], fv[kHeld ? kS : 1];
        __syncthreads();                                   // with whoever still reads from the buffers
        if (threadIdx.x == 0) not_finite = 0;
        if constexpr (kHeld) {                             // through the buffers of the stages
            char* const second = kH == 2 ? pool + kStage : pool;
            fetch_tile(pool, t.k, gk);
            if (kH == 2) fetch_tile(second, t.v, gv);
            arrive();
            take_columns<T, D>(fk, pool + in_tile, all_places.along);
            if (kH == 1) {
                arrive();
                fetch_tile(second, t.v, gv);
                arrive();
            }
            take_columns<T, D>(fv, second + in_tile, all_places.along);
            arrive();
        } else {
            fetch_tile(tile, t.k, gk);
            fetch_tile(tile + kTile * L::kLine, t.v, gv);
        }
        if (n) issue(pool, 0);
        int cut = 0;
        f32x16 dk[kU], dv[kU];
        // Scores; do v^T beside their exponentials; dv's sums beside the gradients of the scores; dk's.
        auto work = [&](const char* b, int i) __attribute__((always_inline)) {
            Places<T, D> places = all_places.again();
            if constexpr (kCuts > 1) places.across ^= cut * kSumCols * (int)sizeof(T);
            const int pair = begin + i * kRows + 32 * half;
            if (kSkip<T> && pair + 32 <= some_see) return;                // all of it is hidden from the wavefront's keys
            const char* sq = b + 32 * half * L::kLine;
            const char* sg = sq + kBytes;
            const char* st = b + 2 * kBytes + 128 * half + 16 * hi;
            constexpr int kN = 2 * kS + 4 * kU, kAhead = sizeof(T) == 4 ? 2 : kHeld ? 4 : 3, kFrom = kS + (sizeof(T) == 4 ? 1 : 2);
            typename L::frag a[kAhead], own[kHeld ? 1 : kAhead];
            typename W::Part c[kAhead];
            auto fetch = [&](auto n) __attribute__((always_inline)) {
                constexpr int j = decltype(n)::value, m = j - 2 * kS;
                if constexpr (j < kS) {
                    a[j % kAhead] = L::along(sq, places.along, j);
                    if constexpr (!kHeld) own[j % kAhead] = L::along(keys, places.along, j);
                } else if constexpr (j < 2 * kS) {
                    a[j % kAhead] = L::along(sg, places.along, j - kS);
                    if constexpr (!kHeld) own[j % kAhead] = L::along(values, places.along, j - kS);
                } else if constexpr (j < kN) {
                    c[j % kAhead] = W::template across<D>(m < 2 * kU ? sg : sq, places.across, m % kU, m / kU % 2);
                }
            };
            f32x16 p = (f32x16)(0.f), ds = (f32x16)(0.f);
            f32x4 lse[2], delta[2];                // four pairs' are read while the four in front of them are worked on
            lse[0] = *(const f32x4*)st;
            static_for<kAhead>([&](auto n) __attribute__((always_inline)) { fetch(n); });
            static_for<2 * kS>([&](auto n) __attribute__((always_inline)) {
                constexpr int j = decltype(n)::value;
                __builtin_amdgcn_sched_barrier(0);
                auto column = [&](auto& held) __attribute__((always_inline)) {
                    if constexpr (kHeld) return held[j % kS];
                    else return own[j % kAhead];
                };
                if constexpr (j < kS) p = multiply(a[j % kAhead], column(fk), p);
                else ds = multiply(a[j % kAhead], column(fv), ds);
                fetch(std::integral_constant<int, j + kAhead>());
                if constexpr (j >= kFrom)
#pragma unroll
                    for (int r = (j - kFrom) * 16 / (2 * kS - kFrom); r < (j - kFrom + 1) * 16 / (2 * kS - kFrom); ++r) {
                        if (r % 4 == 0 && r < 12) lse[(r / 4 + 1) % 2] = *(const f32x4*)(st + 32 * (r / 4 + 1));
                        p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[r], t.scale_log2, -lse[r / 4 % 2][r % 4]));
                    }
            });
            __builtin_amdgcn_sched_barrier(0);
            W wp(p);
            const char* sd = st + 256;
            if (pair < all_see) {
                asm volatile("");              // a branch, as above
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f32x4 less = *(const f32x4*)(sd + 32 * i);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const bool here = pair + 8 * i + 4 * hi + e >= least;
                        ds[4 * i + e] = here ? p[4 * i + e] * (ds[4 * i + e] - less[e]) : 0.f;
                        p[4 * i + e] = here ? p[4 * i + e] : 0.f;
                    }
                }
                wp = W(p);
#pragma unroll
                for (int r = 0; r < 16; ++r) p[r] = 1.f;           // what follows leaves ds as it is
                sd = zeros + 16 * hi;
            }
            delta[0] = *(const f32x4*)sd;
            static_for<2 * kU>([&](auto n) __attribute__((always_inline)) {
                constexpr int j = decltype(n)::value;
                dv[j % kU] = W::add(c[(j + 2 * kS) % kAhead], wp.part[j / kU], dv[j % kU]);
                fetch(std::integral_constant<int, j + 2 * kS + kAhead>());
#pragma unroll
                for (int r = j * 8 / kU; r < (j + 1) * 8 / kU; ++r) {
                    if (r % 4 == 0 && r < 12) delta[(r / 4 + 1) % 2] = *(const f32x4*)(sd + 32 * (r / 4 + 1));
                    ds[r] = p[r] * (ds[r] - delta[r / 4 % 2][r % 4]);
                }
                __builtin_amdgcn_sched_barrier(0);
            });
            const W ws(ds);
            static_for<2 * kU>([&](auto n) __attribute__((always_inline)) {
                constexpr int j = decltype(n)::value;
                dk[j % kU] = W::add(c[(j + 2 * kS + 2 * kU) % kAhead], ws.part[j / kU], dk[j % kU]);
                fetch(std::integral_constant<int, j + 2 * kS + 2 * kU + kAhead>());
                __builtin_amdgcn_sched_barrier(0);
            });
        };
        auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int c = 0; c < kU; ++c) dk[c] = dv[c] = (f32x16)(0.f);
        };
        for (; cut < kCuts; ++cut) {
            if (cut) {
                __syncthreads();
                if (n) issue(pool, 0);
            }
            clear();
            if (n) stages(n, pool, kStage, issue, work);
            if (!n) __syncthreads();                       // the stages have theirs
            if (t.causal && live && !(all_finite(dk) && all_finite(dv))) not_finite = 1;
            __syncthreads();
            if (not_finite) {
                clear();
                for (int i = 0; i < n; ++i) {
                    const int pair = begin + i * kRows;
                    __syncthreads();
                    issue(pool, i);
                    arrive();
                    if (pair < all_see_here) {
                        const int count = min(32 * half + 32, pairs - pair);
                        add_not_finite<T, D, kSumCols>(pool, cut * kSumCols, 32 * half, count, dk, [&](int j) { return pair + j >= least; });
                        add_not_finite<T, D, kSumCols>(pool + kBytes, cut * kSumCols, 32 * half, count, dv, [&](int j) { return pair + j >= least; });
                        __syncthreads();
                        drop_not_finite<T, kBytes, NT>(pool);
                        drop_not_finite<T, kBytes, NT>(pool + kBytes);
                        __syncthreads();
                    }
                    work(pool, i);
                }
                __syncthreads();
            }
            add_halves<kU, kH>(pool, half, wave, dk);
            if (kH == 2) __syncthreads();
            add_halves<kU, kH>(pool, half, wave, dv);
            const int column = cut * kSumCols, cols = t.cols - column;
            if (!live || half || cols <= 0) continue;
            if (first_stage > 0 || last_stage < seq.stages) {
                float* part = part_place<true>(t, block, first_stage == 0) + (int64_t)(key - first) * t.cols;
                store_columns<float, kSumCols>(part + column, cols, dk, 1.f);
                store_columns<float, kSumCols>(part + kTile * t.cols + column, cols, dv, 1.f);
            } else {
                store_columns<T, kSumCols>((T*)t.dk + at * t.lddk + head * t.cols + column, cols, dk, t.scale);
                store_columns<T, kSumCols>((T*)t.dv + at * t.lddv + head * t.cols + column, cols, dv, 1.f);
            }
        }
    }
}

// ---- parts, joined in their order -------------------------------------------------------------
// kJoinRows rows of the tile in which run number blockIdx.x / (kTile / kJoinRows) + 1 begins, if it is the first one to do so.  A part is `sums` matrices: dq, or dk and dv.
constexpr int kJoinRows = 32;
template <typename T, bool KEYS>
__device__ __forceinline__ void join_tile(const HopAttentionTask& t, int most) {
    constexpr int kSums = KEYS ? 2 : 1, kEach = kJoinRows;
    const Runs runs(KEYS ? t.k_plan : t.q_plan, t.k_heads, most);
    const int64_t run = blockIdx.x / (kTile / kEach) + 1, tiles = runs.plan->tiles;
    if (run >= runs.blocks) return;
    const Place at = begin_of_run(runs, run);
    if (at.stage <= 0) return;
    const int head = (int)(at.tile / tiles), first = blockIdx.x % (kTile / kEach) * kEach;
    const PlanTile seq = tile_of(runs, at.tile - head * tiles);
    int64_t b0, b1;
    if (!runs_inside(runs, head, seq, &b0, &b1) || b0 != run) return;
    const int all = (KEYS ? seq.nk : seq.nq * t.group) - seq.first, rows = min(kEach, all - first);
    auto columns = [&](auto width) __attribute__((always_inline)) {
        constexpr int kWidth = decltype(width)::value;
        typedef float sum __attribute__((ext_vector_type(kWidth)));
        typedef sum sum_any __attribute__((aligned(4)));
        const int per_row = t.cols / kWidth;
        for (int i = threadIdx.x; i < rows * per_row * kSums; i += 256) {
            const int r = i / (per_row * kSums), j = i - r * per_row * kSums, which = KEYS && j >= per_row, c = (j - which * per_row) * kWidth, in = first + r, n = seq.first + in;
            const int64_t place = (int64_t)which * kTile * t.cols + in * t.cols + c;
            sum v = *(const HOPL_GLOBAL sum_any*)(part_place<KEYS>(t, b0 - 1, true) + place);
#pragma unroll 4
            for (int64_t b = b0; b <= b1; ++b) v += *(const HOPL_GLOBAL sum_any*)(part_place<KEYS>(t, b, false) + place);
            T* to;
            if constexpr (KEYS) {
                to = (which ? (T*)t.dv + (seq.k0 + n) * t.lddv : (T*)t.dk + (seq.k0 + n) * t.lddk) + head * t.cols + c;
            } else {
                const int row = hopa_divide(n, t.group_inverse, t.group_shift);
                to = (T*)t.dq + (int64_t)(seq.q0 + row) * t.lddq + (head * t.group + n - row * t.group) * t.cols + c;
            }
            const float by = which ? 1.f : t.scale;
            if constexpr (kWidth == 4) store4(to, 4, v * by);
            else *(HOPL_GLOBAL T*)to = (T)(v[0] * by);
        }
    };
    if (t.cols % 4 == 0) columns(std::integral_constant<int, 4>());
    else columns(std::integral_constant<int, 1>());
}
template <typename T>
__global__ __launch_bounds__(256) void attention_grad_join_kernel(HopAttentionTask t, int most) {
    if (blockIdx.y) join_tile<T, true>(t, most);
    else join_tile<T, false>(t, most);
}

template <typename T, int D>
int launch(const HopAttentionTask& t, const HopAttentionPlan& plan, hipStream_t stream) {
    constexpr int grid = kCus, kThreads = 256 * kHalves<T, D>, kJoins = (kCus - 1) * (kTile / kJoinRows);
    attention_plan_kernel<<<dim3(2), dim3(kPlanners), 0, stream>>>(t, 32 * kHalves<T, D>, plan.q_tiles, plan.k_tiles);
    if (t.q_rows) attention_dq_kernel<T, D><<<dim3(grid), dim3(kThreads), 0, stream>>>(t);
    if (t.k_rows) attention_dkv_kernel<T, D><<<dim3(grid), dim3(kThreads), 0, stream>>>(t);
    attention_grad_join_kernel<T><<<dim3(kJoins, 2), dim3(256), 0, stream>>>(t, grid);
    return (int)hipGetLastError();
}

template <typename T>
int launch(const HopAttentionTask& t, const HopAttentionPlan& plan, hipStream_t stream) {
    launch_copies<T>(plan.copies, stream);
    return t.cols <= 64 ? launch<T, 64>(t, plan, stream) : launch<T, 128>(t, plan, stream);
}

}  // namespace

HopAttentionPlan hopa_grad_plan(HopAttentionTask* task, int dtype, char* scratch) {
    HopAttentionTask& t = *task;
    HopAttentionPlan p = {};
    Planner planner(task, &p, dtype, scratch);
    p.q_tiles = ((int64_t)t.q_rows * t.group + kTile - 1) / kTile + t.S;
    p.k_tiles = ((int64_t)t.k_rows + kTile - 1) / kTile + t.S;
    auto plan_bytes = [](int64_t tiles) { return sizeof(Plan) + tiles * sizeof(PlanTile); };
    const int heads = t.k_heads * t.group;
    t.terms = (float*)planner.take((size_t)2 * heads * t.q_rows * 4);
    t.q_plan = planner.take(plan_bytes(p.q_tiles));
    t.k_plan = planner.take(plan_bytes(p.k_tiles));
    t.partial = (float*)planner.take((size_t)kCus * 2 * 3 * kTile * t.cols * 4);          // two parts of a workgroup, of dq, dk and dv
    planner.align(t.q, t.ldq, t.q_rows, heads, t.q_begin);
    planner.align(t.grad, t.ldgrad, t.q_rows, heads, t.q_begin);
    planner.align(t.o, t.ldo, t.q_rows, heads, t.q_begin);
    planner.align(t.k, t.ldk, t.k_rows, t.k_heads, t.k_begin);
    planner.align(t.v, t.ldv, t.k_rows, t.k_heads, t.k_begin);
    return p;
}

int hopa_grad(const HopAttentionTask& t, int dtype, const HopAttentionPlan& plan, void* stream) {
    return dtype == HOP_BF16 ? launch<bf16>(t, plan, (hipStream_t)stream) : launch<float>(t, plan, (hipStream_t)stream);
}
