// libpatconv: attention of many query rows over the paged cache of 8 bits, on the 5th-generation tensor cores (sm_100a).
//
// A block takes 128 rows (query rows times the query heads of one key head), one to a thread, and goes through their tokens 64 at
// a time.  Tensor memory holds the scores [128][64] and the sums [128][dim]:
//   * scores: kind::i8, the queries' bytes (two, fp32 three, see attention.cu) against the key codes as they lie in the cache, one
//     accumulator per byte; a thread reads its row's 64 integers and has its softmax without any exchange;
//   * probabilities go to shared memory as fp16 (fp32: in two parts), value codes are widened to fp16 there, rows of tokens being the
//     contiguous direction (the operand is given as transposed), and kind::f16 adds their product to the sums.
// The sums are rescaled only where a row's largest product of probability and scale rises by more than 2^7: what goes into fp16
// is lifted by 2^7, so that it holds what that leaves (attention.cuh).
// A warp of its own copies the codes, two steps ahead, and issues the matrix instructions, the product of step j and the scores of step
// j + 1 back to back; meanwhile the threads widen the values of step j + 1.  They meet that warp alone (barriers in shared memory), not
// one another.  Two blocks to an SM fill each other's gaps.
//
// The work is cut into equal pieces as in attention.cu; units are counted tile by tile here, since a causal tile of an early row takes
// few of them.
//
// Bound by the matrix units and the exponentials about alike (a unit of dim 128: 128 x 64 x 128 twice at 8192 multiply-adds a clock,
// scores in two integer products at twice that, 256 clocks in all; 8192 exponentials at 16 a clock, 512 clocks).
#include "attention.cuh"
#include "ptx.cuh"

namespace attention {
using patconv::fence_async_proxy;
using patconv::mbar_init;
using patconv::mbar_wait;
using patconv::mma_f16;
using patconv::mma_i8;
using patconv::operand_desc;
using patconv::tc_commit;
using patconv::tc_fence_after;
using patconv::tc_fence_before;
using patconv::tmem_alloc;
using patconv::tmem_free;
using patconv::tmem_ld16;
using patconv::tmem_st16;
using patconv::tmem_wait_ld;
using patconv::tmem_wait_st;

constexpr int kRowWarps = kWideRows / 32, kW = kRowWarps + 1;      // warps that own rows; the last one copies and issues

template <int DT, int D> struct Wide {
    static constexpr bool SPLIT = DT == XGEN_F32;
    static constexpr int TERMS = SPLIT ? 3 : 2;
    static constexpr int CODES = kWideUnit * D;           // of keys, or values
    static constexpr int Q = TERMS * kWideRows * D;
    static constexpr int VALUES = kWideUnit * D * 2;
    static constexpr int PROBS = kWideRows * kWideUnit * 2;
    static constexpr int SHARED = Q + 4 * CODES + VALUES + PROBS * (SPLIT ? 2 : 1);
    static constexpr int COLUMNS = TERMS * kWideUnit + D <= 256 ? 256 : 512;
    // The matrix unit rounds sums toward zero, and each of a unit's 8 products adds to what is lost: sums over 25 units were off by
    // 1.8e-6 on average, in one direction.  fp32 layers add up FOLD units at a time, and the totals apart: in tensor memory
    // where there is room, else in the workspace.  Root mean square errors, and us for 2 x 1024 rows over 5000 tokens, dim 128: 2.3e-6 and
    // 515 without, 6.9e-7 and 528 by fours, 5.1e-7 and 543 by twos; dim 64 (workspace) 1.4e-6 and 296, 7.0e-7 and 330, 5.0e-7 and 368.
    // fp16 layers 64: over 262144 tokens as one sum their values were short of two fp16 steps.  (The same sizes, dim 128: 308 without, 312.)
    static constexpr bool FOLD_NEAR = TERMS * kWideUnit + 2 * D <= COLUMNS;
    static constexpr int FOLD = !SPLIT ? 64 : FOLD_NEAR ? 2 : 4;
    // Sums of two terms lose their lowest bits, so that what is left goes into 23: at most one unit of what is left, 2^DROP/32512 of what the
    // query row's largest component times a key step gives, and up to 0.75 of a unit, the same for a page, in the subtraction that follows:
    // 1/145 (1/73) in all (fp16 queries would have up to 16 steps' worth in a sum of 128).
    static constexpr int DROP = D <= 128 ? 7 : 8;
    static constexpr int BLOCKS = COLUMNS == 256 && SHARED <= 104 * 1024 ? 2 : 1;
};

// What a sequence asks for, and a tile of its rows.
struct WideSequence { int row, n, length, end, tiles; };
struct WideTile { int from, to, units; };                 // tokens [from, to) that some row sees
__device__ __forceinline__ WideSequence wide_sequence(const RunParams &P, int s) {
    const Span sp = span_of(P.batch, s);
    WideSequence q;
    q.row = sp.row; q.n = sp.n;
    q.length = length_of(P.batch, s);
    q.end = (int)min((int64_t)q.length, P.batch.table_stride * P.cache.page_tokens);
    if (P.launched > 1 && q.n * P.group <= kNarrowMost) q.n = 0;
    if (q.end < q.length && q.n > 0) atomicExch(P.status, 1);
    q.tiles = (int)(((int64_t)q.n * P.group + kWideRows - 1) / kWideRows);
    return q;
}
__device__ __forceinline__ WideTile wide_tile(const RunParams &P, const WideSequence &q, int tile) {
    const int before = q.length - q.n, row0 = tile * kWideRows, row1 = min(q.n * P.group, row0 + kWideRows) - 1;
    WideTile t;
    t.from = P.window > 0 ? max(max(before + row0 / P.group, 0) - P.window + 1, 0) & ~15 : 0;
    t.to = max(min(before + row1 / P.group + 1, q.end), t.from);
    t.units = max((t.to - t.from + kWideUnit - 1) / kWideUnit, 1);
    return t;
}

template <int DT, int D> __global__ void __launch_bounds__(kWideThreads, Wide<DT, D>::BLOCKS) wide_kernel(const RunParams P) {
    using T = typename Elem<DT>::T;
    using W = Wide<DT, D>;
    constexpr int TERMS = W::TERMS, CHUNKS = D / 16;
    extern __shared__ __align__(128) unsigned char shared[];
    int8_t *const qs = reinterpret_cast<int8_t *>(shared);                  // [TERMS][128 rows][D], 8 rows of 16 bytes contiguous
    unsigned char *const codes = shared + W::Q;                             // [2 stages][keys, values][64 tokens][D], likewise
    unsigned char *const values = codes + 4 * W::CODES;                     // fp16 [8 tokens of 16 bytes][D/8][8]
    unsigned char *const probs = values + W::VALUES;                        // fp16 [128 rows][64 tokens], 8 rows of 16 bytes contiguous
    __shared__ float stage_scale[2][2][4];                                  // [stage][keys, values][16 tokens]
    __shared__ float4 stage_value[2][4];                                    // of the values' scales: exponent, kLift plus log2 of the rest, reciprocal of both
    __shared__ unsigned stage_there[2];                                     // which 16 tokens of a stage are in pages that are there (bits 0-3), with a lost scale (4-7)
    __shared__ int64_t units_of[kWideSequences];                            // of a key head
    __shared__ int64_t scan[kW + 1], start_units;
    __shared__ int start_s, start_tile, start_unit;
    __shared__ __align__(8) uint64_t bars[6];
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int H = P.cache.heads, G = P.group, worker = blockIdx.x;
    const uint32_t bar_s = smem_at(&bars[0]), bar_o = smem_at(&bars[1]), bar_p = smem_at(&bars[2]), bar_c = smem_at(&bars[3]), bar_end = smem_at(&bars[5]);
    wait_before();

    // ---- this block's piece of the line of units: sequences, key heads, tiles, units
    int64_t todo, skipped = 0, first_unit;
    WideSequence q;
    int s, head, tile;
    {
        const int S = P.batch.sequences;
        for (int i = warp; i < S; i += kW) {
            const WideSequence w = wide_sequence(P, i);
            int64_t u = 0;
            for (int t = lane; t < w.tiles; t += 32) u += wide_tile(P, w, t).units;
#pragma unroll
            for (int d = 16; d; d >>= 1) u += __shfl_xor_sync(~0u, u, d);
            if (lane == 0) units_of[i] = u;
        }
        if (tid == 0) {
            scan[0] = 0;
            s_abort = 0;
            mbar_init(bar_s, 1);
            mbar_init(bar_o, 1 + P.extra);
            mbar_init(bar_p, kWideRows);
            mbar_init(bar_c, 32);
            mbar_init(bar_c + 8, 32);
            mbar_init(bar_end, 1);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncthreads();
        const int each = (S + kWideThreads - 1) / kWideThreads, s0 = min(tid * each, S), s1 = min(s0 + each, S);
        int64_t own = 0;
        for (int i = s0; i < s1; ++i) own += H * units_of[i];
        int64_t upto = own;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int64_t v = __shfl_up_sync(~0u, upto, d);
            if (lane >= d) upto += v;
        }
        if (lane == 31) scan[warp + 1] = upto;
        __syncthreads();
        int64_t before = upto - own, all = 0;
#pragma unroll
        for (int w = 0; w < kW; ++w) {
            if (w < warp) before += scan[w + 1];
            all += scan[w + 1];
        }
        const int64_t piece = max(quotient(all + P.workers - 1, P.workers), (int64_t)1), from = piece * worker;
        todo = min(piece, all - from);
        if (todo > 0 && before <= from && from < before + own) {
            int64_t left = from - before;
            for (int i = s0; i < s1; ++i) {
                const int64_t u = H * units_of[i];
                if (left < u) { start_s = i; start_units = left; break; }
                left -= u;
            }
        }
        __syncthreads();
        if (todo <= 0) {
            if (tid == 0) P.cut[worker].units = 0;
            return;
        }
        s = start_s;
        q = wide_sequence(P, s);
        head = (int)quotient(start_units, units_of[s]);
        if (warp == 0) {
            int64_t left = start_units - head * units_of[s];
            for (int t0 = 0; t0 < q.tiles; t0 += 32) {
                const int u = t0 + lane < q.tiles ? wide_tile(P, q, t0 + lane).units : 0;
                int sum = u;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const int v = __shfl_up_sync(~0u, sum, d);
                    if (lane >= d) sum += v;
                }
                const unsigned hit = __ballot_sync(~0u, left < sum);
                if (hit) {
                    const int at = __ffs(hit) - 1;
                    if (lane == at) { start_tile = t0 + at; start_unit = (int)left - (sum - u); }
                    break;
                }
                left -= __shfl_sync(~0u, sum, 31);
            }
        }
        __syncthreads();
        tile = start_tile;
        skipped = start_unit;
        first_unit = from - skipped;
        if (tid == 0) {
            Cut c;
            c.first = first_unit; c.piece = piece;
            c.units = wide_tile(P, q, tile).units; c.row = q.row; c.n = q.n; c.head = head; c.row0 = tile * kWideRows;
            P.cut[worker] = c;
        }
    }

    // ---- tensor memory (not before the launch ahead is done: it may want all of it)
    if (warp == kRowWarps) {
        tmem_alloc<false>(smem_at(&s_tmem), W::COLUMNS);
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = s_tmem, my_lanes = (uint32_t)(warp * 32) << 16, t_scores = tmem, t_sums = tmem + TERMS * kWideUnit;
    int *const timeout = P.status + 1;
    // Whether it came, the same for the whole warp.  A warp whose wait runs out copies, issues and writes no more: so do the others' waits for it,
    // soon after, and the block ends once the matrix instructions that are under way have.
    const auto wait = [&](uint32_t bar, uint32_t parity) {
        const bool came = __all_sync(~0u, mbar_wait<false>(bar, parity, &s_abort, timeout, P.limit_us));
        tc_fence_after();
        return came;
    };
    bool stop = false;
    int phase_s = 0, phase_o = 0, phase_p = 0, phase_c = 0;      // (phase_c counts steps: two barriers in turn)
    constexpr uint32_t IDESC_S = ((uint32_t)(kWideUnit >> 3) << 17) | (8u << 24) | (2u << 4) | (1u << 7) | (1u << 10);      // s8 s8 -> s32
    constexpr uint32_t IDESC_O = ((uint32_t)(D >> 3) << 17) | (8u << 24) | (1u << 4) | (1u << 16);                          // f16 f16 (transposed) -> f32
    const uint64_t q_desc = operand_desc(smem_at(qs), 128, D * 8), k_desc = operand_desc(smem_at(codes), 128, D * 8);
    const uint64_t p_desc = operand_desc(smem_at(probs), 128, kWideUnit * 16), v_desc = operand_desc(smem_at(values), D * 16, 128);

    // this thread's totals, 16 at a time: (times `since`) plus r, or r alone
    float4 *const fold = P.fold + (int64_t)worker * (D / 4) * kWideRows + tid;
    const auto add_totals = [&](int c, uint32_t (&r)[16], float since) {
        if constexpr (W::FOLD_NEAR) {
            uint32_t t[16];
            tmem_ld16(t_sums + D + my_lanes + c * 16, t);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 16; ++i) r[i] = __float_as_uint(fmaf(__uint_as_float(t[i]), since, __uint_as_float(r[i])));
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float4 t = fold[(c * 4 + i) * kWideRows];
                const float four[4] = {t.x, t.y, t.z, t.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) r[4 * i + j] = __float_as_uint(fmaf(four[j], since, __uint_as_float(r[4 * i + j])));
            }
        }
    };
    const auto keep_totals = [&](int c, const uint32_t (&r)[16]) {
        if constexpr (W::FOLD_NEAR) tmem_st16(t_sums + D + my_lanes + c * 16, r);
        else
#pragma unroll
            for (int i = 0; i < 4; ++i)
                fold[(c * 4 + i) * kWideRows] = make_float4(__uint_as_float(r[4 * i]), __uint_as_float(r[4 * i + 1]), __uint_as_float(r[4 * i + 2]), __uint_as_float(r[4 * i + 3]));
    };

    bool whole = skipped == 0;
    int slot = 0;
    while (todo > 0) {
        const WideTile w = wide_tile(P, q, tile);
        const int row0 = tile * kWideRows, rows = min(kWideRows, q.n * G - row0), before = q.length - q.n;
        const int units = (int)min(todo, (int64_t)(w.units - skipped));
        const bool last_part = skipped + units == w.units;
        float l = 0.0f, m = -INFINITY, unit = -INFINITY, since = 1.0f;       // since: what the totals are to be multiplied by
        if (warp == kRowWarps) {
            // ---- codes, two steps ahead; matrix instructions, whenever the threads are done with a step (first: with the queries)
            const int token_begin = w.from + (int)skipped * kWideUnit;
            // lane l < 4 holds the page table's entry of the next step's l-th 16 tokens
            const auto entry_of = [&](int token) {
                const int at = (token + lane * 16) >> P.cache.page_shift;
                return lane < 4 && token + lane * 16 < w.to && at < P.batch.table_stride ? P.batch.table[(int64_t)s * P.batch.table_stride + at] : -2;
            };
            int entry = entry_of(token_begin), fetched = 0;
            const uint32_t my_place = smem_at(codes) + (lane & 7) * 16;
            const auto fetch = [&] {
                if (fetched < units) {
                    const int stage = (phase_c + fetched) & 1, token = token_begin + fetched * kWideUnit;
                    const bool good = entry >= 0 && entry < P.cache.pages;
                    if (entry != -2 && !good) atomicExch(P.status, 1);
                    const unsigned there = __ballot_sync(~0u, good) & 15u;
                    if (lane == 0) stage_there[stage] = there;
                    const int64_t page = (int64_t)entry * H + head;
                    const int64_t first = ((page << P.cache.page_shift) + ((token + lane * 16) & (P.cache.page_tokens - 1))) * D;      // of this lane's 16 tokens
                    if (good) {
                        copy_async4(smem_at(&stage_scale[stage][0][lane]), P.cache.scale[0] + page);
                        copy_async4(smem_at(&stage_scale[stage][1][lane]), P.cache.scale[1] + page);
                    }
                    const uint32_t place0 = my_place + stage * 2 * W::CODES;
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const int64_t from = __shfl_sync(~0u, first, g) + (lane & 7) * D + (lane >> 3) * 16;
                        if (!(there >> g & 1)) continue;
                        const int8_t *const k = P.cache.codes[0] + from, *const v = P.cache.codes[1] + from;
#pragma unroll
                        for (int i = 0; i < 2 * ((CHUNKS + 3) / 4); ++i) {                 // 8 tokens x 4 pieces of 16 bytes at a time
                            const int block = i & 1, c = (i >> 1) * 4 + (lane >> 3);
                            const uint32_t place = place0 + (2 * g + block) * (D * 8) + c * 128;
                            if (CHUNKS % 4 && c >= CHUNKS) continue;
                            copy_async16(place, k + block * 8 * D + (i >> 1) * 64);
                            copy_async16(place + W::CODES, v + block * 8 * D + (i >> 1) * 64);
                        }
                    }
                    ++fetched;
                    entry = entry_of(token + kWideUnit);
                }
                copy_async_commit();
            };
            const uint32_t q_hi = (uint32_t)(q_desc >> 32), k_hi = (uint32_t)(k_desc >> 32), p_hi = (uint32_t)(p_desc >> 32), v_hi = (uint32_t)(v_desc >> 32);
            fetch();
            fetch();
            for (int u = -1; u < units; ++u) {
                if (u + 1 < units) {                      // the next step's codes are there
                    if (u < 0) copy_async_wait<1>(); else copy_async_wait<0>();
                    const int stage = (phase_c + u + 1) & 1;
                    __syncwarp();                         // (lane 0 wrote it)
                    const unsigned there = stage_there[stage];
                    const float v = lane < 4 && there >> lane & 1 ? stage_scale[stage][1][lane] : 0.0f;      // (what this lane copied itself)
                    const unsigned lost = __ballot_sync(~0u, !(v < INFINITY));
                    if (lane < 4) {
                        const Split f = split_scale(v);
                        stage_value[stage][lane] = make_float4(f.e, (float)kLift + log2f(f.f), pow2(-kLift) / f.f, 0.0f);
                    }
                    if (lost && lane == 0) stage_there[stage] = there | lost << 4;
                    fence_async_proxy();
                    patconv::mbar_arrive(bar_c + 8 * stage);
                }
                if (!wait(bar_p, phase_p++ & 1)) { stop = true; break; }
                if (lane == 0) {
                    if (u >= 0) {
#pragma unroll
                        for (int k = 0; k < kWideUnit / 16; ++k)
#pragma unroll
                            for (int part = W::SPLIT ? 1 : 0; part >= 0; --part)
                                mma_f16<false>(t_sums, (uint32_t)p_desc + part * (W::PROBS / 16) + k * 16, p_hi, (uint32_t)v_desc + k * 2 * D, v_hi, IDESC_O,
                                               u % W::FOLD > 0 || k > 0 || part != (W::SPLIT ? 1 : 0));
                        tc_commit<false>(bar_o, 0);
                    }
                    if (u + 1 < units) {
                        const uint32_t b0 = (uint32_t)k_desc + ((phase_c + u + 1) & 1) * 2 * W::CODES / 16;
#pragma unroll
                        for (int c = 0; c < D / 32; ++c)
#pragma unroll
                            for (int k = 0; k < TERMS; ++k)
                                mma_i8<false>(t_scores + k * kWideUnit, (uint32_t)q_desc + k * (kWideRows * D / 16) + c * 16, q_hi, b0 + c * 16, k_hi, IDESC_S, c > 0);
                        tc_commit<false>(bar_s, 0);
                    }
                }
                __syncwarp();
                if (u >= 0) fetch();                      // into the stage that this step leaves
            }
            phase_c += units;
        } else {
            // ---- queries: a thread copies its row's bytes (where there is no row, the last one's: what comes of it goes nowhere)
            const int my_row = row0 + min(tid, rows - 1);
            const int64_t flat = (int64_t)head * P.batch.rows * G + (int64_t)q.row * G + my_row;
            const float factor = P.q_factor[flat];
            {
                const int8_t *const from = P.q_bytes + flat * (TERMS * D);
                const uint32_t to = smem_at(qs) + (tid >> 3) * (D * 8) + (tid & 7) * 16;
#pragma unroll
                for (int k = 0; k < TERMS; ++k)
#pragma unroll
                    for (int c = 0; c < CHUNKS; ++c) copy_async16(to + k * kWideRows * D + c * 128, from + k * D + c * 16);
                copy_async_commit();
                copy_async_wait<0>();
            }
            const auto hand_over = [&] {                  // what this thread wrote is the matrix instructions'
                fence_async_proxy();
                tc_fence_before();
                patconv::mbar_arrive(bar_p);
            };
            const int token_begin = w.from + (int)skipped * kWideUnit;
            hand_over();
            const int position = before + my_row / G;
#pragma unroll 1
            for (int u = 0; u < units; ++u) {
                const int stage = phase_c & 1, token = token_begin + u * kWideUnit;
                if (!wait(bar_c + 8 * stage, phase_c++ >> 1 & 1)) { stop = true; break; }
                const unsigned there = stage_there[stage] & 15u, lost = stage_there[stage] >> 4;
                float k_scale[4];
#pragma unroll
                for (int g = 0; g < 4; ++g) k_scale[g] = stage_scale[stage][0][g];
                // Of 16 tokens each: what is added to a score so that its power of two is the product of probability and scale, lifted; what the
                // sum of these is multiplied by to be one of probabilities; the score from which on references go up.  What is 2^-45 of the
                // reference or less is nothing in fp16, wherever below that it is put, but its probability counts.
                // Scores are less m in fp32 layers (in the rounding that they have anyway); in fp16 layers, where that took 3 % longer, m is in
                // what is added, rounded down: far from 0, where that is by many units, a product must not come out above 2^15.
                float off[4], plain[4], limit[4], base;
                const auto prepare = [&] {
                    base = m == -INFINITY ? 0.0f : m;
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const float4 value = stage_value[stage][g];
                        const float far = fminf(fmaxf(value.x - unit, -45.0f), 110.0f), reach = kFar + fminf(unit - value.x, 0.0f);
                        off[g] = W::SPLIT ? far + value.y : __fadd_rd(far + value.y, -base);
                        plain[g] = exp2_approx(-far) * value.z;
                        limit[g] = !W::SPLIT ? __fadd_rd(m, reach) : m == -INFINITY ? -INFINITY : reach;
                    }
                };
                prepare();
                // ---- values to fp16
                {
                    const unsigned char *const from = codes + stage * 2 * W::CODES + W::CODES;
                    constexpr int MINE = kWideUnit * CHUNKS / kWideRows;
                    uint4 raw[MINE];                      // (all loads ahead of all stores, which could alias for all the compiler knows)
#pragma unroll
                    for (int i = 0; i < MINE; ++i) {
                        const int p = tid + kWideRows * i, block = (p >> 3) / CHUNKS, c = (p >> 3) % CHUNKS;
                        raw[i] = *reinterpret_cast<const uint4 *>(from + block * (D * 8) + c * 128 + (p & 7) * 16);
                    }
                    if (u > 0 && !wait(bar_o, phase_o++ & 1)) { stop = true; break; }       // the product before: values, probabilities and sums are free
                    if (u > 0 && u % W::FOLD == 0) {
#pragma unroll 1
                        for (int c = 0; c < D / 16; ++c) {
                            uint32_t r[16];
                            tmem_ld16(t_sums + my_lanes + c * 16, r);
                            tmem_wait_ld();
                            if (u > W::FOLD) add_totals(c, r, since);
                            keep_totals(c, r);
                        }
                        if (W::FOLD_NEAR) tmem_wait_st();
                        since = 1.0f;
                    }
#pragma unroll
                    for (int i = 0; i < MINE; ++i) {
                        const int p = tid + kWideRows * i, block = (p >> 3) / CHUNKS, c = (p >> 3) % CHUNKS;
                        const uint4 r = raw[i];
                        const uint32_t x[4] = {r.x ^ 0x80808080u, r.y ^ 0x80808080u, r.z ^ 0x80808080u, r.w ^ 0x80808080u};
                        uint4 *const to = reinterpret_cast<uint4 *>(values + block * (D * 16) + c * 256 + (p & 7) * 16);
                        to[0] = make_uint4(widen_codes<0x4140>(x[0]), widen_codes<0x4342>(x[0]), widen_codes<0x4140>(x[1]), widen_codes<0x4342>(x[1]));
                        to[8] = make_uint4(widen_codes<0x4140>(x[2]), widen_codes<0x4342>(x[2]), widen_codes<0x4140>(x[3]), widen_codes<0x4342>(x[3]));
                    }
                }
                // ---- scores in powers of two
                if (!wait(bar_s, phase_s++ & 1)) { stop = true; break; }
                float sc[kWideUnit];
                constexpr int TOGETHER = TERMS == 3 ? 1 : 2;      // (loads are waited for all at once)
                uint32_t rr[TOGETHER][TERMS][16];
#pragma unroll
                for (int c = 0; c < kWideUnit / 16; ++c) {
                    if (c % TOGETHER == 0) {
#pragma unroll
                        for (int j = 0; j < TOGETHER; ++j)
#pragma unroll
                            for (int k = 0; k < TERMS; ++k) tmem_ld16(t_scores + my_lanes + k * kWideUnit + (c + j) * 16, rr[j][k]);
                        tmem_wait_ld();
                    }
                    const uint32_t (&r)[TERMS][16] = rr[c % TOGETHER];
                    if constexpr (TERMS == 3) {
                        const float by = k_scale[c] * factor;
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            sc[c * 16 + i] = fmaf(fmaf((float)(int)r[2][i], 65536.0f, (float)((int)r[1][i] * 256 + (int)r[0][i])), by, -base);
                    } else {
                        // an integer of less than 23 bits as the low bits of 1.5 * 2^23 (a conversion would take the exponentials' unit)
                        const float by = k_scale[c] * factor * (float)(1 << W::DROP), less = -12582912.0f * by;
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            sc[c * 16 + i] = fmaf(__uint_as_float(0x4B400000u + ((int)r[0][i] >> W::DROP) + (r[1][i] << (8 - W::DROP))), by, less);
                    }
                }
                if (__any_sync(~0u, token + kWideUnit - 1 > position || token <= position - P.window && P.window > 0) || there != 15u) {
                    // tokens [first, last] of the step, as bits; 16 at a time where a page is not there
                    const int last = position - token, first = P.window > 0 ? last - P.window + 1 : 0;
                    uint64_t seen = last >= kWideUnit - 1 ? ~0ull : last < 0 ? 0ull : (2ull << last) - 1;
                    if (first > 0) seen = first >= kWideUnit ? 0ull : seen & ~0ull << first;
                    uint32_t half[2] = {(uint32_t)seen, (uint32_t)(seen >> 32)};
#pragma unroll
                    for (int g = 0; g < 4; ++g)
                        if (!(there >> g & 1)) half[g >> 1] &= g & 1 ? 0xFFFFu : 0xFFFF0000u;
#pragma unroll
                    for (int i = 0; i < kWideUnit; ++i) sc[i] = half[i >> 5] & 1u << (i & 31) ? sc[i] : -INFINITY;
                }
                float most[4];
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    most[g] = max_or_nan(sc[16 * g], sc[16 * g + 1]);
#pragma unroll
                    for (int i = 2; i < 16; i += 2) most[g] = max_or_nan(most[g], sc[16 * g + i], sc[16 * g + i + 1]);
                }
                // ---- the row's references go up; a NaN goes into l (what the row does not see has a score of -infinity)
                float shrink = 1.0f;
                if (__any_sync(~0u, most[0] > limit[0] || most[1] > limit[1] || most[2] > limit[2] || most[3] > limit[3])) {
                    const float largest = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
                    float heaviest = -INFINITY;
                    if constexpr (W::SPLIT) {
                        const bool first = m == -INFINITY;
                        float up = 0.0f;
                        if (largest > (first ? -INFINITY : kFar)) {
                            up = raise_reference(m, base, largest);
                            if (!first) l *= exp2_approx(-up);
                            unit -= up;
                        }
#pragma unroll
                        for (int i = 0; i < kWideUnit; ++i) sc[i] -= up;
#pragma unroll
                        for (int g = 0; g < 4; ++g)
                            if (most[g] - up > -100.0f) heaviest = fmaxf(heaviest, most[g] - up + stage_value[stage][g].x);
                    } else {
                        if (largest > m + kFar) {
                            const float to = ceilf(largest);
                            l *= exp2_approx(m - to);
                            unit -= to - m;
                            m = to;
                        }
#pragma unroll
                        for (int g = 0; g < 4; ++g)
                            if (most[g] - m > -100.0f) heaviest = fmaxf(heaviest, most[g] - m + stage_value[stage][g].x);
                    }
                    if (heaviest > unit + kFar) {
                        const float to = ceilf(heaviest);
                        shrink = exp2_approx(unit - to);
                        unit = to;
                    }
                    prepare();
                }
                if (lost) {                               // the rows that see some of a lost page are lost, the others are not
#pragma unroll
                    for (int g = 0; g < 4; ++g)
                        if (lost >> g & 1 && !(most[g] == -INFINITY)) l = NAN;
                }
                // ---- products of probabilities and scales, lifted; totals are of the probabilities alone
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    uint32_t hi[8], lo[8];
                    float sum0 = 0.0f, sum1 = 0.0f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float x0 = exp2_approx(sc[16 * g + 2 * i] + off[g]), x1 = exp2_approx(sc[16 * g + 2 * i + 1] + off[g]);
                        sum0 += x0;
                        sum1 += x1;
                        hi[i] = pack_half(x0, x1);
                        if (W::SPLIT) {
                            const __half2 h = *reinterpret_cast<const __half2 *>(&hi[i]);
                            lo[i] = pack_half(x0 - __low2float(h), x1 - __high2float(h));
                        }
                    }
                    l = fmaf(sum0 + sum1, plain[g], l);
                    uint4 *const to = reinterpret_cast<uint4 *>(probs + (tid >> 3) * (kWideUnit * 16) + g * 256 + (tid & 7) * 16);
                    to[0] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                    to[8] = make_uint4(hi[4], hi[5], hi[6], hi[7]);
                    if (W::SPLIT) {
                        to[W::PROBS / 16] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                        to[W::PROBS / 16 + 8] = make_uint4(lo[4], lo[5], lo[6], lo[7]);
                    }
                }
                since *= shrink;
                if (u % W::FOLD > 0 && __any_sync(~0u, shrink != 1.0f)) {
#pragma unroll 1
                    for (int c = 0; c < D / 16; ++c) {
                        uint32_t r[16];
                        tmem_ld16(t_sums + my_lanes + c * 16, r);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 16; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * shrink);
                        tmem_st16(t_sums + my_lanes + c * 16, r);
                    }
                    tmem_wait_st();
                }
                hand_over();
            }
            if (!stop) stop = !wait(bar_o, phase_o++ & 1);
        }
        todo -= units;

        if (warp < kRowWarps && !stop) {
            // ---- the tile's results: a row to a thread
            const bool complete = whole && last_part;
            const float2 f = complete ? result_factors(l, unit) : make_float2(1.0f, 1.0f);
            T *const y = static_cast<T *>(P.y) + (int64_t)(q.row + (row0 + tid) / G) * P.y_stride + (int64_t)(head * G + (row0 + tid) % G) * D;
            float *const part = P.partial + (((int64_t)worker * 2 + slot) * kWideRows + tid) * D;
#pragma unroll 1
            for (int c = 0; c < D / 16; ++c) {
                uint32_t r[16];
                tmem_ld16(t_sums + my_lanes + c * 16, r);
                tmem_wait_ld();
                if (units > W::FOLD) add_totals(c, r, since);
                if (tid < rows) {
                    float x[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[i] = f.x == 0.0f ? 0.0f : __uint_as_float(r[i]) * f.x * f.y;
                    if (!complete) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) reinterpret_cast<float4 *>(part + c * 16)[i] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
                    } else {
                        T o[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[i] = narrow<T>(x[i]);
                        if (P.vec_y) {
                            uint4 raw[sizeof(T)];
                            memcpy(raw, o, sizeof o);
#pragma unroll
                            for (int i = 0; i < (int)sizeof(T); ++i) reinterpret_cast<uint4 *>(y + c * 16)[i] = raw[i];
                        } else {
#pragma unroll
                            for (int i = 0; i < 16; ++i) y[c * 16 + i] = o[i];
                        }
                    }
                }
                __syncwarp();
            }
            if (!complete) P.stats[((int64_t)worker * 2 + slot) * kWideRows + tid] = make_float4(m, l, unit, 0.0f);
        }
        tc_fence_before();
        stop = __syncthreads_or(stop);
        tc_fence_after();
        if (stop) break;
        if (todo > 0) {
            skipped = 0;
            if (++tile >= q.tiles) {
                tile = 0;
                if (++head >= H) {
                    head = 0;
                    do q = wide_sequence(P, ++s); while (q.n == 0);
                }
            }
            whole = true;
            slot = 1;
        }
    }
    let_next();
    copy_async_wait<0>();
    if (stop && warp == kRowWarps) {
        if (lane == 0) tc_commit<false>(bar_end, 0);
        __syncwarp();
        wait(bar_end, 0);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kRowWarps) tmem_free<false>(tmem, W::COLUMNS);
}

// The queries of all rows, turned, as a factor times integers: a warp takes a row and some of its heads, which share their angles; a lane four
// neighbouring pairs of a head, so that D/8 lanes make up a head and bytes leave four at a time.
template <int DT, int D> __global__ void __launch_bounds__(kQueryThreads) query_kernel(const RunParams P) {
    using T = typename Elem<DT>::T;
    constexpr int TERMS = Wide<DT, D>::TERMS, LANES = D <= 32 ? 4 : D <= 64 ? 8 : D <= 128 ? 16 : 32, AT_ONCE = 32 / LANES;
    const int lane = threadIdx.x & 31, in_head = lane % LANES, G = P.group, heads = P.cache.heads * G;
    let_next();
    wait_before();
    const int per_row = (heads + kQueryHeads - 1) / kQueryHeads;
    const int64_t warp = (int64_t)blockIdx.x * (kQueryThreads / 32) + (threadIdx.x >> 5);
    const int64_t row = warp / per_row;
    if (row >= P.batch.rows) return;
    const int head0 = (int)(warp - row * per_row) * kQueryHeads, head1 = min(head0 + kQueryHeads, heads);
    const int s = sequence_of_row(P.batch, row);
    if (s < 0) return;
    const Span sp = span_of(P.batch, s);
    if (row < sp.row || (P.launched > 1 && sp.n * G <= kNarrowMost)) return;
    const int position = length_of(P.batch, s) - sp.n + (int)(row - sp.row);       // (below 0: nothing will be seen)
    const T *const from = static_cast<const T *>(P.q) + row * P.q_stride;
    // pairs u0 .. u0 + 3: components at x .. x + 3 and y .. y + 3 (halves), or x .. x + 7; any way where the rotation ends inside
    const int u0 = 4 * in_head, pairs = P.rotation.rotary / 2;
    const bool in = u0 < D / 2, halves = pairs > 0 && !P.rotation.interleaved;
    const bool apart = halves && u0 < pairs, any = halves && pairs % 4;
    const int x = apart ? u0 : 2 * u0, y = apart ? u0 + pairs : 2 * u0 + 4;
    float2 by[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) by[j] = in && u0 + j < pairs ? angle(P.rotation.freq[u0 + j], max(position, 0)) : make_float2(1.0f, 0.0f);
#pragma unroll 2
    for (int head2 = head0; head2 < head1; head2 += AT_ONCE) {
        const int head = head2 + lane / LANES;
        const bool there = in && head < head1;
        const auto component = [&](int j) {               // of the lane's eight: firsts of the pairs, then seconds
            if (any) {
                const int2 at = pair_of(P.rotation, u0 + (j & 3));
                return j < 4 ? at.x : at.y;
            }
            return apart ? (j < 4 ? x + j : y + j - 4) : 2 * (u0 + (j & 3)) + (j >> 2);
        };
        float v[8];
        float largest = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = there ? widen(from[head * D + component(j)]) : 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            turn(by[j], v[j], v[4 + j]);
            largest = max_or_nan(largest, fabsf(v[j]), fabsf(v[4 + j]));
        }
#pragma unroll
        for (int d = 1; d < LANES; d <<= 1) largest = max_or_nan(largest, __shfl_xor_sync(~0u, largest, d));
        // (as in narrow_kernel)
        constexpr float LIMIT = TERMS == 3 ? 127.0f * 65536.0f : 127.0f * 256.0f;
        const bool finite = largest < INFINITY;
        const float top = fmaxf(largest, 7.8886e-31f), scale = finite ? LIMIT / top : 0.0f;
        if (!there) continue;
        const int64_t flat = ((int64_t)(head / G) * P.batch.rows + row) * G + head % G;
        int8_t *const to = P.q_bytes + flat * (TERMS * D);
        uint32_t bytes[TERMS][2];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            int n = finite ? min(max(__float2int_rn(v[j] * scale), -(int)LIMIT), (int)LIMIT) : 0;
            // where the four are to leave together, their places in the word: halves in order, neighbours alternating
            const int word = apart ? j >> 2 : (j & 3) >> 1, place = apart ? j & 3 : 2 * (j & 1) + (j >> 2);
#pragma unroll
            for (int k = 0; k < TERMS; ++k) {              // lowest byte first
                const int low = k == TERMS - 1 ? n : (int)(int8_t)n;
                if (any) to[k * D + component(j)] = (int8_t)low;
                if (j == 0) bytes[k][0] = bytes[k][1] = 0;
                bytes[k][word] |= (uint32_t)(low & 255) << (8 * place);
                n = (n - low) >> 8;
            }
        }
        if (!any) {
#pragma unroll
            for (int k = 0; k < TERMS; ++k) {
                *reinterpret_cast<uint32_t *>(to + k * D + x) = bytes[k][0];
                *reinterpret_cast<uint32_t *>(to + k * D + y) = bytes[k][1];
            }
        }
        if (in_head == 0) P.q_factor[flat] = finite ? top / LIMIT * P.scale : NAN;
    }
}

template <int DT, int D> static WideKernel wide_of() {
    using W = Wide<DT, D>;
    if constexpr (W::SHARED > 216 * 1024) return {};
    else return {(const void *)wide_kernel<DT, D>, (const void *)query_kernel<DT, D>, W::SHARED, W::BLOCKS, W::TERMS, !W::FOLD_NEAR};
}
template <int DT> static WideKernel wide_dt(int dim) {
    switch (dim) {
    case 32: return wide_of<DT, 32>();
    case 64: return wide_of<DT, 64>();
    case 96: return wide_of<DT, 96>();
    case 128: return wide_of<DT, 128>();
    case 192: return wide_of<DT, 192>();
    default: return wide_of<DT, 256>();
    }
}
WideKernel wide_kernel_for(xgen_dtype t, int dim) { return t == XGEN_F32 ? wide_dt<XGEN_F32>(dim) : wide_dt<XGEN_F16_F32ACC>(dim); }

}  // namespace attention
