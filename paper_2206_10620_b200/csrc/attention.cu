// libpatconv: a paged key/value cache of 8 bits and attention over it, for sm_100a, and their C ABI.
//
// append  one block per page that new tokens reach, some heads, and keys or values: a head's new entries stay in registers as fp32
//         (turned there, if keys) until their largest magnitude has decided the page's scale.  A token's angle is that of the page's first token, worked
//         out once for each of a thread's pairs, and that of its slot, from a table made with the handle.
// read    codes times scales; blocks as for append, 16 bytes of the result a thread at a time.
// run     `narrow_kernel`: few query rows (with all query heads of a key head) against the whole cache of a sequence, bound
//         by the cache's bytes.  The work of a call is a line of units (64 tokens of one key head, for one tile of rows), cut into
//         equal pieces, one for each block that the GPU holds at once; where a cut falls inside a tile's tokens the pieces
//         leave partial results, which `combine_kernel` joins in their order.  So any mixture of lengths fills the GPU evenly.
//         Sequences of many rows are wide_kernel's, in attention_wide.cu, cut and joined the same way.
// Scores are exact integer products: a query row is a factor times integers of 16 bits (fp32: 24), split into two (three) signed
// bytes, and integer matrix instructions multiply each with the key codes as they lie in the cache.  Values meet probabilities
// in fp16 (fp32: in two parts): a code is exact there, widened by byte permutes and one subtraction.  The page's scales are
// applied to scores and probabilities in fp32; attention.cuh says relative to what the latter become fp16.
#include <cmath>
#include <climits>
#include <cstring>
#include <new>
#include <vector>

#include "attention.cuh"

struct xgen_attention_packed {
    xgen_attention_desc d;
    int device, sms;
    int workers[2];             // blocks of narrow_kernel that the device holds at once, for one eight of rows and two
    int wide_workers;           // blocks of wide_kernel, or 0 where there is none
    uint64_t *d_freq;           // [rotary/2] turns per position, as 64-bit fractions; behind them the cosines and sines of the slots of a page
    int *d_status;
    int extra_arrivals;         // see xgen_attention_test_expect_arrivals
};

namespace attention {

// Tokens of one page that a batch's rows are.
struct PagePart {
    int64_t page;                     // -1: not there
    int row, n, slot, first;          // first of the rows, number of them, slot of the first; position of the page's first token
};
// Page number `want` of those that the batch's rows reach, sequence by sequence; false where there are fewer.  Every lane of the warp takes part.
__device__ __forceinline__ bool find_page(const Batch &B, const Cache &C, int want, PagePart &part) {
    const int lane = threadIdx.x & 31, PT = C.page_tokens;
    int seq = -1, page_at = 0;
    int64_t before = 0;
    for (int i0 = 0; i0 < B.sequences; i0 += 32) {
        const int i = i0 + lane;
        int first = 0, count = 0;
        if (i < B.sequences) {
            const int n = span_of(B, i).n, length = length_of(B, i);
            const int p0 = max(length - n, 0);
            if (n > 0 && length > p0) { first = p0 >> C.page_shift; count = ((length - 1) >> C.page_shift) - first + 1; }
        }
        int upto = count;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int v = __shfl_up_sync(~0u, upto, d);
            if (lane >= d) upto += v;
        }
        const unsigned hit = __ballot_sync(~0u, want < before + upto);
        if (hit) {
            const int at = __ffs(hit) - 1;
            seq = i0 + at;
            page_at = __shfl_sync(~0u, first, at) + (int)(want - before) - (__shfl_sync(~0u, upto, at) - __shfl_sync(~0u, count, at));
            break;
        }
        before += __shfl_sync(~0u, upto, 31);
    }
    if (seq < 0) return false;
    const Span sp = span_of(B, seq);
    const int length = length_of(B, seq);
    const int lo = max(max(length - sp.n, 0), page_at * PT);
    const int hi = (int)min((int64_t)length, (int64_t)(page_at + 1) * PT);
    part.n = hi - lo; part.slot = lo - page_at * PT; part.first = page_at * PT;
    part.row = sp.row + (lo - (length - sp.n));
    part.page = page_of(B, C, seq, lo);
    return true;
}

// ---- append ------------------------------------------------------------------------------------------------------------------
struct AppendParams {
    Batch batch;
    Cache cache;
    Rotation rotation;
    const void *in[2];
    int64_t stride;
    int dim, room, heads;       // tokens that a block can hold, heads that it takes
    bool vec[2];
    int *status;
};

constexpr int kAppendMost = 512;      // threads of a block: as many as it takes for ITEMS items each
// ITEMS: items of 8 pairs (16 components of a token) that a thread holds.

// How a thread's items of a token lie: two pieces of 8 neighbours, next to each other or (a half's and the other half's) apart, or any way.
enum Lay { PLAIN, HALVES, PAIRS, ANY };

// Heads [head0, head1) of the page.  Item i of thread `tid` is pairs 8 s .. 8 s + 7 of token tid / per_token + i * (threads / per_token), s =
// tid % per_token (the number of threads is a multiple of per_token).
template <int DT, int LAY, int ITEMS> __device__ __forceinline__ void append_heads(const AppendParams &P, const PagePart &part, int which, int head0, int head1) {
    using T = typename Elem<DT>::T;
    __shared__ unsigned most_bits[2][kAppendMost / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x;
    const int H = P.cache.heads, D = P.dim, PT = P.cache.page_tokens, R = P.rotation.rotary, pairs = R / 2;
    const int per_token = D / 16, s = tid % per_token, token0 = tid / per_token, step = threads / per_token;
    const bool turned = LAY == ANY ? which == 0 && R > 0 : LAY != PLAIN;
    const bool apart = LAY == PLAIN || (LAY == HALVES ? 16 * s < R : LAY == ANY && turned && !P.rotation.interleaved && 16 * s < R);
    const int at0 = apart ? 8 * s : 16 * s, at1 = apart ? 8 * s + (LAY == PLAIN ? D / 2 : pairs) : 16 * s + 8;          // (not in ANY)
    float2 base[8];                                       // of this thread's pairs at the page's first token
    if (turned) {
#pragma unroll
        for (int j = 0; j < 8; ++j) base[j] = 8 * s + j < pairs ? angle(P.rotation.freq[8 * s + j], part.first) : make_float2(1.0f, 0.0f);
    }
    const T *const in = static_cast<const T *>(P.in[which]) + (int64_t)(part.row + token0) * P.stride;
    constexpr int W = sizeof(T) / 2;                      // 16-byte pieces of 8 components
    uint4 raw[ITEMS][2 * W];
    const auto ask = [&](int head) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const T *const from = in + (int64_t)(i * step) * P.stride + head * D;
            const bool there = token0 + i * step < part.n;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                raw[i][w] = there ? reinterpret_cast<const uint4 *>(from + at0)[w] : make_uint4(0, 0, 0, 0);
                raw[i][W + w] = there ? reinterpret_cast<const uint4 *>(from + at1)[w] : make_uint4(0, 0, 0, 0);
            }
        }
    };
#pragma unroll 1
    for (int head = head0; head < head1; ++head) {
        // ---- the new entries in fp32
        float v[ITEMS][16];
        if (LAY != ANY) ask(head);
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const T *const from = in + (int64_t)(i * step) * P.stride + head * D;
            const bool there = token0 + i * step < part.n;
            if (LAY == ANY) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {             // (in `apart` order, or neighbours)
                    const int2 at = apart ? pair_of(P.rotation, 8 * s + j) : make_int2(16 * s + 2 * j, 16 * s + 2 * j + 1);
                    const float x = there ? widen(from[at.x]) : 0.0f, y = there ? widen(from[at.y]) : 0.0f;
                    if (apart) { v[i][j] = x; v[i][8 + j] = y; }
                    else { v[i][2 * j] = x; v[i][2 * j + 1] = y; }
                }
            }
        }
        float *const scale_at = P.cache.scale[which] + part.page * H + head;
        const float was = part.slot ? *scale_at : 0.0f;
        float largest = 0.0f;                             // magnitude; as bits, a NaN is above infinity
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            if (LAY != ANY) {
#pragma unroll
                for (int w = 0; w < 2 * W; ++w) {
                    const uint32_t u[4] = {raw[i][w].x, raw[i][w].y, raw[i][w].z, raw[i][w].w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        if (DT == XGEN_F32) v[i][4 * w + k] = __uint_as_float(u[k]);
                        else {
                            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&u[k]));
                            v[i][(8 * w + 2 * k) & 15] = f.x;
                            v[i][(8 * w + 2 * k + 1) & 15] = f.y;
                        }
                    }
                }
            }
            if (turned && token0 + i * step < part.n) {
                const float2 *const by_slot = P.rotation.slots + (part.slot + token0 + i * step) * pairs + 8 * s;
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (8 * s + j < pairs) {
                        const float2 o = __ldg(by_slot + j), b = base[j];
                        const float2 by = make_float2(b.x * o.x - b.y * o.y, b.y * o.x + b.x * o.y);
                        if (apart) turn(by, v[i][j], v[i][8 + j]);
                        else turn(by, v[i][2 * j], v[i][2 * j + 1]);
                    }
            }
#pragma unroll
            for (int j = 0; j < 16; ++j) largest = max_or_nan(largest, fabsf(v[i][j]));
        }
        unsigned most = __reduce_max_sync(~0u, __float_as_uint(largest));
        if (lane == 0) most_bits[head & 1][warp] = most;
        __syncthreads();
        for (int i = 0; i < threads / 32; ++i) most = max(most, most_bits[head & 1][i]);
        const float amax = __uint_as_float(most);

        // ---- the scale
        float scale = was;
        int halvings = 0;
        if (most >= 0x7F800000u || isnan(was)) scale = NAN;
        else if (!(was > 0.0f)) {
            scale = most ? fmaxf(amax / 127.0f, 1.17549435e-38f) : 0.0f;
            halvings = 100;                               // older entries are 0
        } else
            while (amax > 127.5f * scale) { scale *= 2.0f; ++halvings; }
        if (tid == 0) *scale_at = scale;

        // ---- codes
        int8_t *const codes = P.cache.codes[which] + (part.page * H + head) * (int64_t)PT * D;
        if (halvings > 0) {
            const float by = pow2(-min(halvings, 100));
            for (int c = tid; c < part.slot * per_token; c += threads) {
                uint4 old = reinterpret_cast<const uint4 *>(codes)[c];
                int8_t q[16];
                memcpy(q, &old, 16);
#pragma unroll
                for (int i = 0; i < 16; ++i) q[i] = (int8_t)__float2int_rn((float)q[i] * by);
                memcpy(&old, q, 16);
                reinterpret_cast<uint4 *>(codes)[c] = old;
            }
        }
        const float by = scale > 0.0f ? 1.0f / scale : 0.0f;
        if (amax * by > 127.4f) {                         // some entry may round beyond 127
            const float most_code = 127.0f * scale;
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
#pragma unroll
                for (int j = 0; j < 16; ++j) v[i][j] = fminf(fmaxf(v[i][j], -most_code), most_code);
        }
        int8_t *const to0 = codes + (int64_t)(part.slot + token0) * D;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            if (token0 + i * step >= part.n) break;
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t q[4];                            // 1.5 * 2^23 added leaves the nearest integer in the lowest bits
#pragma unroll
                for (int k = 0; k < 4; ++k) {             // (the quotient itself, by its residual after Markstein: some entries lie halfway between two codes)
                    const float x = v[i][4 * j + k], about = x * by;
                    q[k] = __float_as_uint(fmaf(fmaf(-about, scale, x), by, about) + 12582912.0f);
                }
                w[j] = __byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410);
            }
            if (isnan(scale)) w[0] = w[1] = w[2] = w[3] = 0;
            int8_t *const to = to0 + i * step * D;
            if (LAY != ANY && apart) {
                *reinterpret_cast<uint2 *>(to + at0) = make_uint2(w[0], w[1]);
                *reinterpret_cast<uint2 *>(to + at1) = make_uint2(w[2], w[3]);
            } else if (LAY == ANY && apart) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int2 at = pair_of(P.rotation, 8 * s + j);
                    to[at.x] = (int8_t)(w[j >> 2] >> (8 * (j & 3)));
                    to[at.y] = (int8_t)(w[2 + (j >> 2)] >> (8 * (j & 3)));
                }
            } else *reinterpret_cast<uint4 *>(to + 16 * s) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
}

template <int DT, int ITEMS> __global__ void __launch_bounds__(kAppendMost, 1) append_kernel(const AppendParams P) {
    const int tid = threadIdx.x, which = blockIdx.z;
    let_next();
    wait_before();

    PagePart part;
    if (!find_page(P.batch, P.cache, blockIdx.x, part)) return;
    if (part.page < 0 || part.n > P.room) {
        if (tid == 0) atomicExch(P.status, 1);
        return;
    }
    const int head0 = blockIdx.y * P.heads, head1 = min(head0 + P.heads, P.cache.heads);
    const int R = which == 0 ? P.rotation.rotary : 0;
    if (!P.vec[which] || (R % 16 && !P.rotation.interleaved)) append_heads<DT, ANY, ITEMS>(P, part, which, head0, head1);
    else if (R == 0) append_heads<DT, PLAIN, ITEMS>(P, part, which, head0, head1);
    else if (P.rotation.interleaved) append_heads<DT, PAIRS, ITEMS>(P, part, which, head0, head1);
    else append_heads<DT, HALVES, ITEMS>(P, part, which, head0, head1);
}

// ---- read --------------------------------------------------------------------------------------------------------------------
struct ReadParams {
    Batch batch;
    Cache cache;
    void *out[2];
    int64_t stride;
    int dim, heads;             // heads that a block takes
    uint32_t token_of;          // 2^32 / (pieces of 16 bytes of a token's head), rounded up: for the token of a piece by one product
    bool vec[2];
    int *status;
};

constexpr int kReadThreads = 256;

template <int DT> __global__ void __launch_bounds__(kReadThreads, 5) read_kernel(const ReadParams P) {
    using T = typename Elem<DT>::T;
    constexpr int E = 16 / sizeof(T), MINE = 4;           // a thread's pieces: MINE at a time, the same of every head
    const int tid = threadIdx.x, H = P.cache.heads, D = P.dim, per_token = D / E;
    let_next();
    wait_before();
    PagePart part;
    if (!find_page(P.batch, P.cache, blockIdx.x, part)) return;
    if (part.page < 0 && tid == 0) atomicExch(P.status, 1);
    const int head0 = blockIdx.y * P.heads, head1 = min(head0 + P.heads, H), pieces = part.n * per_token;
    const int64_t page_codes = ((part.page * H << P.cache.page_shift) + part.slot) * D, next_head = (int64_t)D << P.cache.page_shift;
#pragma unroll 1
    for (int piece0 = tid; piece0 < pieces; piece0 += kReadThreads * MINE) {
        int from[MINE];
        int64_t to[MINE];
#pragma unroll
        for (int i = 0; i < MINE; ++i) {
            const int piece = piece0 + i * kReadThreads, token = (int)__umulhi((uint32_t)piece, P.token_of), at = piece * E;
            from[i] = at;
            to[i] = (int64_t)(part.row + token) * P.stride + (at - token * D);
        }
#pragma unroll 1
        for (int both = 2 * head0; both < 2 * head1; ++both) {
            const int w = both & 1, head = both >> 1;
            const float scale = part.page < 0 ? 0.0f : P.cache.scale[w][part.page * H + head];
            const int8_t *const codes = P.cache.codes[w] + page_codes + head * next_head;
            T *const out = static_cast<T *>(P.out[w]) + head * D;
            uint32_t raw[MINE][E / 4];
#pragma unroll
            for (int i = 0; i < MINE; ++i) {
#pragma unroll
                for (int j = 0; j < E / 4; ++j) raw[i][j] = 0;
                if (part.page >= 0 && piece0 + i * kReadThreads < pieces) {
                    if (E == 8) {
                        const uint2 u = *reinterpret_cast<const uint2 *>(codes + from[i]);
                        raw[i][0] = u.x;
                        raw[i][E / 4 - 1] = u.y;
                    } else raw[i][0] = *reinterpret_cast<const uint32_t *>(codes + from[i]);
                }
            }
#pragma unroll
            for (int i = 0; i < MINE; ++i) {
                if (piece0 + i * kReadThreads >= pieces) break;
                T v[E];
#pragma unroll
                for (int j = 0; j < E / 4; ++j) {
                    const uint32_t u = raw[i][j] ^ 0x80808080u, h[2] = {widen_codes<0x4140>(u), widen_codes<0x4342>(u)};
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h[k]));
                        if constexpr (DT == XGEN_F32) {
                            v[4 * j + 2 * k] = f.x * scale;
                            v[4 * j + 2 * k + 1] = f.y * scale;
                        } else {
                            const __half2 o = __floats2half2_rn(f.x * scale, f.y * scale);
                            memcpy(&v[4 * j + 2 * k], &o, 4);
                        }
                    }
                }
                if (P.vec[w]) {
                    uint4 o;
                    memcpy(&o, v, 16);
                    *reinterpret_cast<uint4 *>(out + to[i]) = o;
                } else {
#pragma unroll
                    for (int j = 0; j < E; ++j) out[to[i] + j] = v[j];
                }
            }
        }
    }
}

// ---- run: few rows against a long cache ------------------------------------------------------------------------------------------
constexpr int kTokens = 16;          // tokens that a warp takes at a time, in one page
constexpr int kWarps = 4, kThreads = 32 * kWarps, kUnit = kWarps * kTokens;
// fp16 layers: units that a tile goes on with the same sums.  The matrix unit rounds them toward zero, 2^-23 at most with every unit: over 4096
// units a row's values were short of an fp16 step, over 16384 of two.  (fp32 layers add up with rounding, at every 16 tokens; as much
// takes one request over 1000 tokens from 10.8 us to 12.9 here.)
constexpr int kUnitsOnce = 512;


// What a sequence asks for: rows, tiles of rows for each key head, units of a tile, where its tokens begin.
struct Sequence {
    int row, n, length, from, tiles, units;
};
template <int ROWS> __device__ __forceinline__ Sequence sequence_of(const RunParams &P, int s) {
    const Span sp = span_of(P.batch, s);
    Sequence q;
    q.row = sp.row; q.n = sp.n;
    // tokens beyond the table's are nobody's
    const int64_t held = P.batch.table_stride * P.cache.page_tokens;
    q.length = length_of(P.batch, s);
    const int end = (int)min((int64_t)q.length, held);
    if (end < q.length && q.n > 0) atomicExch(P.status, 1);
    const int first = max(q.length - q.n, 0);             // the first row's position, if it has one
    q.from = P.window > 0 && first - P.window + 1 > 0 ? (first - P.window + 1) / kTokens * kTokens : 0;
    if (P.launched > 1 && q.n * P.group > kNarrowMost) q.n = 0;        // another kernel's
    q.tiles = (int)(((int64_t)q.n * P.group + ROWS - 1) / ROWS);
    q.units = q.n > 0 ? max((end - q.from + kUnit - 1) / kUnit, 1) : 0;
    return q;
}

// A place on the line of units: unit `unit` of tile `tile` (of key head `head`) of sequence `s`.
struct Place {
    Sequence q;
    int s, head, tile, unit;
};
template <int ROWS> __device__ __forceinline__ void next_place(const RunParams &P, Place &c) {
    if (++c.unit < c.q.units) return;
    c.unit = 0;
    if (++c.tile < c.q.tiles) return;
    c.tile = 0;
    if (++c.head < P.cache.heads) return;
    c.head = 0;
    do {
        if (++c.s >= P.batch.sequences) return;
        c.q = sequence_of<ROWS>(P, c.s);
    } while (c.q.n == 0);
}

__device__ __forceinline__ uint32_t turn_matrix(uint32_t v) {        // an 8 x 8 matrix of 16-bit elements, transposed
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
// DT: type.  D: components of a head.  NT: eights of query rows in a tile.  Tokens are the rows of the score product and query rows its
// columns, so a tile of up to eight rows (all that a decoding step has of most models) wastes no more than its empty columns.
template <int DT, int D, int NT> struct Narrow {
    static constexpr bool SPLIT = DT == XGEN_F32;          // probabilities of 22 bits as two of 11
    static constexpr int TERMS = SPLIT ? 3 : 2;            // bytes of a query component
    static constexpr int ROWS = 8 * NT;
    static constexpr bool Q_IN_REGISTERS = TERMS * NT * D <= 512;
    static constexpr int ROW = D + 16;                     // bytes of a token's codes in shared memory: 8 tokens meet no bank twice
    static constexpr int STAGES = D <= 64 ? 4 : D <= 128 ? 3 : 2;
    static constexpr int STAGE = 2 * kTokens * ROW;        // keys, values
    static constexpr int Q_ROW = D + 16;                   // bytes of a query row's term
    static constexpr int Q_BYTES = TERMS * ROWS * Q_ROW;
    static constexpr int RING = kWarps * STAGES * STAGE;
    static constexpr int SUM_ROW = D + 4;
    static constexpr int SUMS = ROWS * SUM_ROW;
    static constexpr int COPIES = NT == 1 ? 2 : 1;         // of the sums, for as many warps at a time
    static constexpr int SHARED = RING + Q_BYTES + COPIES * SUMS * 4;
    static constexpr int BLOCKS = D <= 128 ? 3 : D * NT <= 256 ? 2 : 1;
};

template <int DT, int D, int NT> __global__ void __launch_bounds__(kThreads, Narrow<DT, D, NT>::BLOCKS) narrow_kernel(const RunParams P) {
    using T = typename Elem<DT>::T;
    using N = Narrow<DT, D, NT>;
    constexpr int ROWS = N::ROWS, TERMS = N::TERMS;
    extern __shared__ __align__(16) unsigned char shared[];
    unsigned char *const ring = shared;
    int8_t *const qs = reinterpret_cast<int8_t *>(shared + N::RING);                     // [TERMS][ROWS][Q_ROW]
    float *const sums = reinterpret_cast<float *>(shared + N::RING + N::Q_BYTES);        // [COPIES][ROWS][SUM_ROW]
    __shared__ float stage_scale[kWarps][N::STAGES][2];
    __shared__ float row_factor[ROWS];
    __shared__ float row_most[kWarps][ROWS], row_total[kWarps][ROWS], row_unit[kWarps][ROWS];
    __shared__ int64_t scan[kWarps + 1], start_units;
    __shared__ int start_s;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const int H = P.cache.heads, G = P.group, worker = blockIdx.x;
    wait_before();

    // ---- this block's piece of the line of units
    int64_t todo;
    Place ahead;
    int64_t skipped;                                       // units of the first tile before the piece
    {
        const int each = (P.batch.sequences + kThreads - 1) / kThreads;
        const int s0 = min(tid * each, P.batch.sequences), s1 = min(s0 + each, P.batch.sequences);
        int64_t own = 0;
        for (int s = s0; s < s1; ++s) {
            const Sequence q = sequence_of<ROWS>(P, s);
            own += (int64_t)H * q.tiles * q.units;
        }
        int64_t upto = own;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int64_t v = __shfl_up_sync(~0u, upto, d);
            if (lane >= d) upto += v;
        }
        if (lane == 31) scan[warp + 1] = upto;
        if (tid == 0) scan[0] = 0;
        __syncthreads();
        int64_t before = upto - own, all = 0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            if (w < warp) before += scan[w + 1];
            all += scan[w + 1];
        }
        const int64_t piece = max(quotient(all + P.workers - 1, P.workers), (int64_t)1);
        const int64_t from = piece * worker;
        todo = min(piece, all - from);
        if (todo > 0 && before <= from && from < before + own) {
            int64_t left = from - before;
            for (int s = s0; s < s1; ++s) {
                const Sequence q = sequence_of<ROWS>(P, s);
                const int64_t u = (int64_t)H * q.tiles * q.units;
                if (left < u) { start_s = s; start_units = left; break; }
                left -= u;
            }
        }
        __syncthreads();
        if (todo <= 0) {
            if (tid == 0) P.cut[worker].units = 0;
            return;
        }
        ahead.s = start_s;
        ahead.q = sequence_of<ROWS>(P, ahead.s);
        const int64_t tile = quotient(start_units, ahead.q.units);
        skipped = start_units - tile * ahead.q.units;
        ahead.unit = (int)skipped;
        ahead.head = (int)quotient(tile, ahead.q.tiles);
        ahead.tile = (int)(tile - (int64_t)ahead.head * ahead.q.tiles);
        if (tid == 0) {
            Cut c;
            c.first = from - skipped; c.piece = piece;
            c.units = ahead.q.units; c.row = ahead.q.row; c.n = ahead.q.n; c.head = ahead.head; c.row0 = ahead.tile * ROWS;
            P.cut[worker] = c;
        }
        // Short pieces: the joining blocks may come as soon as there is room, and find their instructions and arguments in time.
        // (With long ones they, and the kernel behind them, would take room on some SMs from the next call's blocks: 64 sequences of up to
        // 8192 tokens one call after the other 188 us, and 130 with the next launch let go at the end.)
        if (piece <= P.early) let_next();
    }

    // ---- tokens on their way: each warp its own
    const uint32_t my_ring = smem_at(ring) + warp * N::STAGES * N::STAGE;
    uint32_t there = 0;                                    // bit i: stage i holds a tile of tokens that somebody may see
    int64_t left_ahead = todo;
    auto token_of = [&](const Place &c) { return c.q.from + c.unit * kUnit + warp * kTokens; };
    auto entry_of = [&](const Place &c) {                  // the page table's entry (asked for one unit before it is needed)
        const int at = token_of(c) >> P.cache.page_shift;
        return token_of(c) < c.q.length && at < P.batch.table_stride ? P.batch.table[(int64_t)c.s * P.batch.table_stride + at] : -2;
    };
    int entry = entry_of(ahead);
    int first_seen, last_seen;                             // tokens that some row of the tile sees
    auto set_seen = [&] {
        const int before = ahead.q.length - ahead.q.n;     // the first row's position
        last_seen = min(ahead.q.length - 1, before + (ahead.tile * ROWS + ROWS - 1) / G);
        first_seen = P.window > 0 ? max(before + ahead.tile * ROWS / G, 0) - P.window + 1 : 0;
    };
    set_seen();
    // this lane's 16-byte pieces of a tile: row (lane + 32 i) / (D/16), column the rest
    const int8_t *const k_codes = P.cache.codes[0] + lane * 16, *const v_codes = P.cache.codes[1] + lane * 16;
    auto fetch = [&](int stage) {
        if (left_ahead > 0) {
            const int token = token_of(ahead);
            there &= ~(1u << stage);
            if (entry >= 0 && entry < P.cache.pages) {
                if (token <= last_seen && token + kTokens > first_seen) {
                    const int64_t at = (int64_t)entry * H + ahead.head;
                    const int64_t from = ((at << P.cache.page_shift) + (token & (P.cache.page_tokens - 1))) * D;
                    const uint32_t to = my_ring + stage * N::STAGE;
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) {
                        const int c = lane + 32 * i, place = c / (D / 16) * N::ROW + c % (D / 16) * 16;
                        copy_async16(to + place, k_codes + from + i * 512);
                        copy_async16(to + kTokens * N::ROW + place, v_codes + from + i * 512);
                    }
                    if (lane < 2) copy_async4(smem_at(&stage_scale[warp][stage][lane]), P.cache.scale[lane] + at);
                    there |= 1u << stage;
                }
            } else if (entry != -2 && lane == 0) atomicExch(P.status, 1);
            if (--left_ahead > 0) {
                if (ahead.unit + 1 < ahead.q.units) ++ahead.unit;
                else {
                    next_place<ROWS>(P, ahead);
                    set_seen();
                }
                entry = entry_of(ahead);
            }
        }
        copy_async_commit();
    };
    Place now = ahead;
#pragma unroll
    for (int i = 0; i < N::STAGES - 1; ++i) fetch(i);

    int stage = 0;
    const uint32_t a_lane = (uint32_t)((lane & 7) + (lane & 8)) * N::ROW + (lane >> 4) * 16;     // this lane's row of four matrices
    bool whole = skipped == 0, held = false;               // held: the partial results' place has what came of the tile's units so far
    int slot = 0;                                          // of the partial results: 0 for the piece's first tile
    while (todo > 0) {
        // ---- one tile of rows: queries, turned, as a factor times integers
        const int row0 = now.tile * ROWS, rows = min(ROWS, now.q.n * G - row0);
        const int first_position = now.q.length - now.q.n;
        constexpr int PAIRS = (D / 2 + 31) / 32, MINE = ROWS / kWarps;
        float v[MINE][2 * PAIRS];
#pragma unroll
        for (int w = 0; w < MINE; ++w) {                   // (all loads first)
            const int r = warp + w * kWarps, i = (row0 + r) / G;
            const T *const q = static_cast<const T *>(P.q) + (int64_t)(now.q.row + i) * P.q_stride + (int64_t)(now.head * G + (row0 + r) % G) * D;
#pragma unroll
            for (int p = 0; p < PAIRS; ++p) {
                const int u = lane + 32 * p;
                const int2 at = pair_of(P.rotation, u);
                const bool in = r < rows && u < D / 2;
                v[w][2 * p] = in ? widen(q[at.x]) : 0.0f;
                v[w][2 * p + 1] = in ? widen(q[at.y]) : 0.0f;
            }
        }
#pragma unroll
        for (int w = 0; w < MINE; ++w) {
            const int r = warp + w * kWarps, i = (row0 + r) / G;
            unsigned most = 0;
            if (r < rows && first_position + i >= 0) {
#pragma unroll
                for (int p = 0; p < PAIRS; ++p) {
                    const int u = lane + 32 * p;
                    if (u < P.rotation.rotary / 2) turn(angle(P.rotation.freq[u], first_position + i), v[w][2 * p], v[w][2 * p + 1]);
                }
            }
#pragma unroll
            for (int p = 0; p < 2 * PAIRS; ++p) most = max(most, __float_as_uint(v[w][p]) & 0x7FFFFFFFu);
            most = __reduce_max_sync(~0u, most);
            // the largest component becomes 127 * 2^8 (2^16); a row below 2^-100 is taken as if it reached that
            constexpr float LIMIT = TERMS == 3 ? 127.0f * 65536.0f : 127.0f * 256.0f;
            const bool finite = most < 0x7F800000u;
            const float top = fmaxf(__uint_as_float(most), 7.8886e-31f), by = finite ? LIMIT / top : 0.0f;
#pragma unroll
            for (int p = 0; p < PAIRS; ++p) {
                const int u = lane + 32 * p;
                if (u < D / 2) {
                    const int2 at = pair_of(P.rotation, u);
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        int x = finite ? min(max(__float2int_rn(v[w][2 * p + j] * by), -(int)LIMIT), (int)LIMIT) : 0;
#pragma unroll
                        for (int m = 0; m < TERMS; ++m) {  // lowest byte first
                            const int low = m == TERMS - 1 ? x : (int)(int8_t)x;
                            qs[(m * ROWS + r) * N::Q_ROW + (j ? at.y : at.x)] = (int8_t)low;
                            x = (x - low) >> 8;
                        }
                    }
                }
            }
            if (lane == 0) row_factor[r] = finite ? top / LIMIT * P.scale : NAN;
        }
        __syncthreads();
        constexpr int KEPT = N::Q_IN_REGISTERS ? D / 32 : 1;
        uint32_t qf[TERMS][NT][KEPT][2];
        auto query = [&](int m, int n, int c, int h) {
            return *reinterpret_cast<const uint32_t *>(qs + (m * ROWS + n * 8 + g) * N::Q_ROW + c * 32 + 16 * h + 4 * t);
        };
        if (N::Q_IN_REGISTERS) {
#pragma unroll
            for (int m = 0; m < TERMS; ++m)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int c = 0; c < KEPT; ++c) { qf[m][n][c][0] = query(m, n, c, 0); qf[m][n][c][1] = query(m, n, c, 1); }
        }
        float factor[NT][2];
        int position[NT][2];                               // of this lane's rows 8 n + 2t and the next; -1 where there is no row
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int r = 8 * n + 2 * t + j;
                factor[n][j] = row_factor[r];
                position[n][j] = r < rows ? first_position + (row0 + r) / G : -1;
            }
        const int least_position = first_position + row0 / G;

        // o[n][c]: components 16c + 2g of rows 8n + 2t and 8n + 2t + 1, then component 16c + 2g + 1 of both
        float o[NT][D / 16][4];
        float m[NT][2], l[NT][2], unit[NT][2];             // (attention.cuh)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            m[n][0] = m[n][1] = unit[n][0] = unit[n][1] = -INFINITY;
            l[n][0] = l[n][1] = 0.0f;
#pragma unroll
            for (int c = 0; c < D / 16; ++c) o[n][c][0] = o[n][c][1] = o[n][c][2] = o[n][c][3] = 0.0f;
        }

        // ---- its tokens, as far as the piece goes
        const int units = (int)min(todo, (int64_t)(N::SPLIT ? now.q.units - now.unit : min(now.q.units - now.unit, kUnitsOnce)));
        const bool last_part = now.unit + units == now.q.units;
        int token = token_of(now);
        for (int u = 0; u < units; ++u, token += kUnit) {
            fetch(stage == 0 ? N::STAGES - 1 : stage - 1);
            copy_async_wait<N::STAGES - 1>();
            __syncwarp();
            if (there >> stage & 1) {
                const uint32_t k_at = my_ring + stage * N::STAGE + a_lane, v_at = k_at + kTokens * N::ROW;
                const float k_scale = stage_scale[warp][stage][0], v_scale = stage_scale[warp][stage][1];
                int dot[TERMS][NT][4] = {};
#pragma unroll
                for (int c = 0; c < D / 32; ++c) {
                    uint32_t a[4];
                    load_matrices(a, k_at + c * 32);
#pragma unroll
                    for (int k = 0; k < TERMS; ++k)
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            if (N::Q_IN_REGISTERS) mma_bytes(dot[k][n], a, qf[k][n][N::Q_IN_REGISTERS ? c : 0][0], qf[k][n][N::Q_IN_REGISTERS ? c : 0][1]);
                            else mma_bytes(dot[k][n], a, query(k, n, c, 0), query(k, n, c, 1));
                        }
                }
                // scores in powers of two less the reference, what a row does not see out of them (rows: g and g + 8 of the tokens)
                const bool all_seen = token + kTokens - 1 <= least_position && P.window == 0;       // (what the rows behind the last one see is no matter)
                const Split value = split_scale(v_scale);
                float s[NT][4], by[NT][2];
                bool rise = false;
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    float base[2], limit[2];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        base[j] = m[n][j] == -INFINITY ? 0.0f : m[n][j];
                        limit[j] = m[n][j] == -INFINITY ? -INFINITY : kFar + fminf(unit[n][j] - value.e, 0.0f);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int j = token + g + 8 * (i >> 1), p = position[n][i & 1];
                        float x = TERMS == 3 ? fmaf((float)dot[TERMS - 1][n][i], 65536.0f, (float)(dot[1][n][i] * 256 + dot[0][n][i]))
                                             : (float)(dot[1][n][i] * 256 + dot[0][n][i]);
                        x = fmaf(x, k_scale * factor[n][i & 1], -base[i & 1]);
                        if (!all_seen && (j > p || (P.window > 0 && j <= p - P.window))) x = -INFINITY;
                        s[n][i] = x;
                        rise |= x > limit[i & 1];
                    }
                }
                const bool lost = !(v_scale < INFINITY);
                if (__any_sync(~0u, rise || lost)) {       // references go up; the rows that see some of a lost page are lost, the others are not
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        float shrink[2];
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            float x = max_or_nan(s[n][j], s[n][2 + j]);
#pragma unroll
                            for (int d = 4; d < 32; d <<= 1) x = max_or_nan(x, __shfl_xor_sync(~0u, x, d));
                            if (lost && !(x == -INFINITY)) l[n][j] = NAN;
                            const bool first = m[n][j] == -INFINITY;
                            if (x > (first ? -INFINITY : kFar)) {
                                const float up = raise_reference(m[n][j], first ? 0.0f : m[n][j], x);
                                if (!first) l[n][j] *= exp2_approx(-up);
                                unit[n][j] -= up;
                                x -= up;
                                s[n][j] -= up;
                                s[n][2 + j] -= up;
                            }
                            const float weight = x > -100.0f ? ceilf(x + value.e) : -INFINITY;
                            shrink[j] = 1.0f;
                            if (weight > unit[n][j] + kFar) {
                                shrink[j] = exp2_approx(unit[n][j] - weight);
                                unit[n][j] = weight;
                            }
                        }
#pragma unroll
                        for (int c = 0; c < D / 16; ++c) {
                            o[n][c][0] *= shrink[0]; o[n][c][1] *= shrink[1]; o[n][c][2] *= shrink[0]; o[n][c][3] *= shrink[1];
                        }
                    }
                }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const float far = value.e - unit[n][j];
                        by[n][j] = far <= 100.0f ? value.f * exp2_approx(far + (float)kLift) : 0.0f;
#pragma unroll
                        for (int i = 0; i < 2; ++i) s[n][2 * i + j] = exp2_approx(s[n][2 * i + j]);
                        l[n][j] += s[n][j] + s[n][2 + j];
                    }
                uint32_t p[NT][2], p_low[NT][2];           // as the second operand: rows (tokens) 2t .. and 2t + 8 .., column (query row) g
#pragma unroll
                for (int n = 0; n < NT; ++n) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float x0 = s[n][2 * i] * by[n][0], x1 = s[n][2 * i + 1] * by[n][1];
                        const uint32_t high = pack_half(x0, x1);
                        p[n][i] = turn_matrix(high);
                        if (N::SPLIT) {
                            const __half2 h = *reinterpret_cast<const __half2 *>(&high);
                            p_low[n][i] = turn_matrix(pack_half(x0 - __low2float(h), x1 - __high2float(h)));
                        }
                    }
                }
#pragma unroll
                for (int c = 0; c < D / 16; c += 2) {
                    uint32_t r[4];
                    load_matrices_turned(r, v_at + c * 16);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t x0 = r[2 * h] ^ 0x80808080u, x1 = r[2 * h + 1] ^ 0x80808080u;
                        const uint32_t a[4] = {widen_codes<0x4240>(x0), widen_codes<0x4341>(x0), widen_codes<0x4240>(x1), widen_codes<0x4341>(x1)};
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            if (N::SPLIT) {                // (the matrix unit rounds sums toward zero: not the running ones of fp32 layers)
                                float x[4] = {};
                                mma16(x, a, p_low[n][0], p_low[n][1]);
                                mma16(x, a, p[n][0], p[n][1]);
#pragma unroll
                                for (int i = 0; i < 4; ++i) o[n][c + h][i] += x[i];
                            } else mma16(o[n][c + h], a, p[n][0], p[n][1]);
                        }
                    }
                }
                __syncwarp();                              // the stage is free again
            }
            stage = stage + 1 == N::STAGES ? 0 : stage + 1;
        }
        todo -= units;
        // ---- the warps' shares together
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) l[n][j] += __shfl_xor_sync(~0u, l[n][j], d);
                if (g == 0) { row_most[warp][8 * n + 2 * t + j] = m[n][j]; row_total[warp][8 * n + 2 * t + j] = l[n][j]; row_unit[warp][8 * n + 2 * t + j] = unit[n][j]; }
            }
        __syncthreads();
        float top[NT][2], total[NT][2], mine[NT][2], top_unit[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int r = 8 * n + 2 * t + j;
                top[n][j] = row_most[0][r];
#pragma unroll
                for (int w = 1; w < kWarps; ++w) top[n][j] = max_or_nan(top[n][j], row_most[w][r]);
                const float base = top[n][j] == -INFINITY ? 0.0f : top[n][j];
                total[n][j] = 0.0f;
                top_unit[n][j] = -INFINITY;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) {
                    total[n][j] += row_total[w][r] * exp2_approx(row_most[w][r] - base);
                    top_unit[n][j] = fmaxf(top_unit[n][j], row_most[w][r] - base + row_unit[w][r]);
                }
                mine[n][j] = unit[n][j] == -INFINITY ? 0.0f : exp2_approx(m[n][j] - base + unit[n][j] - top_unit[n][j]);
            }
        for (int w = 0; w < kWarps / N::COPIES; ++w) {
            if (warp / N::COPIES == w) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int c = 0; c < D / 16; ++c)
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            float2 *const at = reinterpret_cast<float2 *>(sums + warp % N::COPIES * N::SUMS + (8 * n + 2 * t + j) * N::SUM_ROW + c * 16 + 2 * g);
                            float2 v = w == 0 ? make_float2(0.0f, 0.0f) : *at;
                            v.x += mine[n][j] * o[n][c][j];
                            v.y += mine[n][j] * o[n][c][2 + j];
                            *at = v;
                        }
            }
            __syncthreads();
        }
        float *const partial = P.partial + ((int64_t)worker * 2 + slot) * ROWS * D;
        float4 *const stats = P.stats + ((int64_t)worker * 2 + slot) * ROWS;
        if (!N::SPLIT && held) {                           // what both count for: row_most[1], [2]
            if (warp == 0 && g == 0) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int r = 8 * n + 2 * t + j;
                        const float4 old = stats[r];
                        const float both = max_or_nan(top[n][j], old.x), base = both == -INFINITY ? 0.0f : both;
                        const float mine = top[n][j] - base + top_unit[n][j], theirs = old.x - base + old.z, unit = fmaxf(mine, theirs);
                        total[n][j] = total[n][j] * exp2_approx(top[n][j] - base) + old.y * exp2_approx(old.x - base);
                        row_most[1][r] = top_unit[n][j] == -INFINITY ? 0.0f : exp2_approx(mine - unit);
                        row_most[2][r] = old.z == -INFINITY ? 0.0f : exp2_approx(theirs - unit);
                        top[n][j] = both;
                        top_unit[n][j] = unit;
                    }
            }
            __syncthreads();
        }
        auto sum_at = [&](int i) {                         // element i of the tile (always the same thread's)
            const int r = i / D, at = r * N::SUM_ROW + i % D;
            const float v = N::COPIES == 1 ? sums[at] : sums[at] + sums[N::SUMS + at];
            return !N::SPLIT && held ? v * row_most[1][r] + partial[i] * row_most[2][r] : v;
        };
        const bool complete = whole && last_part;
        if (complete) {
            if (warp == 0 && g == 0) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const float2 f = result_factors(total[n][j], top_unit[n][j]);
                        row_total[0][8 * n + 2 * t + j] = f.x;
                        row_unit[0][8 * n + 2 * t + j] = f.y;
                    }
            }
            __syncthreads();
            for (int i = tid; i < rows * D; i += kThreads) {
                const int r = i / D, row = (row0 + r) / G, head = now.head * G + (row0 + r) % G;
                const float by = row_total[0][r];
                static_cast<T *>(P.y)[(int64_t)(now.q.row + row) * P.y_stride + (int64_t)head * D + i % D] =
                    narrow<T>(by == 0.0f ? 0.0f : sum_at(i) * by * row_unit[0][r]);
            }
        } else {
            for (int i = tid; i < rows * D; i += kThreads) partial[i] = sum_at(i);
            if (warp == 0 && g == 0) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        stats[8 * n + 2 * t + j] = make_float4(top[n][j], total[n][j], top_unit[n][j], 0.0f);
            }
        }
        __syncthreads();
        held = !last_part;
        if (held) now.unit += units;                       // on with the tile, if there is anything to do
        else if (todo > 0) {                               // on to the next tile of rows
            now.unit = now.q.units - 1;
            next_place<ROWS>(P, now);
            whole = true;
            slot = 1;
        }
    }
    let_next();
    copy_async_wait<0>();
}

// Joins the partial results of the tile that the cut before `worker` falls into, if that is the tile's first cut: four groups of threads
// take the parts in turn.
constexpr int kCombineThreads = 512, kGroups = 4, kGroup = kCombineThreads / kGroups, kCombineRows = 16;      // rows of a block
template <int DT, int D, int ROWS> __global__ void __launch_bounds__(kCombineThreads) combine_kernel(const RunParams P) {
    using T = typename Elem<DT>::T;
    constexpr int MINE = ROWS < kCombineRows ? ROWS : kCombineRows;
    __shared__ float4 row_stat[MINE];                     // reference, unit, the sums' two factors
    __shared__ float4 shares[kGroups - 1][kGroup];
    const int worker = blockIdx.x + 1, first_row = blockIdx.y * MINE, tid = threadIdx.x;
    let_next();
    wait_before();
    const Cut c = P.cut[worker];
    const int64_t from = c.piece * worker;
    if (c.units == 0 || c.first == from || c.first < from - c.piece) return;      // no piece; the cut is between two tiles, or not the tile's first
    const int rows = min(MINE, c.n * P.group - c.row0 - first_row);      // of this block's
    if (rows <= 0) return;
    const int parts = (int)quotient(c.first + c.units - 1, c.piece) - (worker - 1) + 1;
    // the first part is its worker's last tile (or all it has), the others are their workers' first
    const int64_t first_slot = (int64_t)(worker - 1) * 2 + (c.first <= from - c.piece ? 0 : 1), next_slot = (int64_t)worker * 2;
    auto slot_of = [&](int part) { return part == 0 ? first_slot : next_slot + 2 * (part - 1); };
    {
        // statistics of a row: some threads of one warp
        constexpr int PER = 32;
        const int r = tid / PER, k = tid % PER;
        if (r < rows) {
            float top = -INFINITY;
            for (int part = k; part < parts; part += PER) top = max_or_nan(top, P.stats[slot_of(part) * ROWS + first_row + r].x);
#pragma unroll
            for (int d = 1; d < PER; d <<= 1) top = max_or_nan(top, __shfl_xor_sync(~0u, top, d));
            const float base = top == -INFINITY ? 0.0f : top;
            float total = 0.0f, unit = -INFINITY;
            for (int part = k; part < parts; part += PER) {
                const float4 x = P.stats[slot_of(part) * ROWS + first_row + r];
                total += exp2_approx(x.x - base) * x.y;
                unit = fmaxf(unit, x.x - base + x.z);
            }
#pragma unroll
            for (int d = 1; d < PER; d <<= 1) {
                total += __shfl_xor_sync(~0u, total, d);
                unit = fmaxf(unit, __shfl_xor_sync(~0u, unit, d));
            }
            const float2 f = result_factors(total, unit);
            if (k == 0) row_stat[r] = make_float4(base, unit, f.x, f.y);
        }
    }
    __syncthreads();
    const auto put = [&](int r, int at, float4 v) {
        const float by = row_stat[r].z, unit = row_stat[r].w;
        T *const to = static_cast<T *>(P.y) + (int64_t)(c.row + (c.row0 + first_row + r) / P.group) * P.y_stride +
                      (int64_t)(c.head * P.group + (c.row0 + first_row + r) % P.group) * D + at;
        const float4 y = by == 0.0f ? make_float4(0.0f, 0.0f, 0.0f, 0.0f) : make_float4(v.x * by * unit, v.y * by * unit, v.z * by * unit, v.w * by * unit);
        to[0] = narrow<T>(y.x); to[1] = narrow<T>(y.y); to[2] = narrow<T>(y.z); to[3] = narrow<T>(y.w);
    };
    const auto add = [&](float4 &v, int part, int r, int at) {
        const int64_t slot = slot_of(part);
        const float4 x = P.stats[slot * ROWS + first_row + r];
        const float4 o = *reinterpret_cast<const float4 *>(P.partial + (slot * ROWS + first_row + r) * D + at);
        const float4 stat = row_stat[r];
        const float f = x.z == -INFINITY ? 0.0f : exp2_approx(x.x - stat.x + x.z - stat.y);
        v.x += f * o.x; v.y += f * o.y; v.z += f * o.z; v.w += f * o.w;
    };
    if (parts <= kGroups) {                               // a thread adds up all parts of what it has
#pragma unroll 2
        for (int i = tid; i < rows * (D / 4); i += kCombineThreads) {
            const int r = i / (D / 4), at = i % (D / 4) * 4;
            float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            for (int part = 0; part < parts; ++part) add(v, part, r, at);
            put(r, at, v);
        }
        return;
    }
    const int group = tid / kGroup, in_group = tid % kGroup;
    for (int i0 = 0; i0 < rows * (D / 4); i0 += kGroup) {
        const int i = i0 + in_group, r = i / (D / 4), at = i % (D / 4) * 4;
        const bool in = r < rows;
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (in) {
#pragma unroll 4
            for (int part = group; part < parts; part += kGroups) add(v, part, r, at);
        }
        if (group) shares[group - 1][in_group] = v;
        __syncthreads();
        if (group == 0 && in) {
#pragma unroll
            for (int k = 0; k < kGroups - 1; ++k) {
                const float4 x = shares[k][in_group];
                v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
            }
            put(r, at, v);
        }
        __syncthreads();
    }
}

// ---- which instance --------------------------------------------------------------------------------------------------------------
struct Kernels {
    const void *narrow, *combine, *combine_wide;
    int shared, rows;
};
template <int DT, int D> static Kernels kernels_of(int nt) {
    if (nt == 1) return {(const void *)narrow_kernel<DT, D, 1>, (const void *)combine_kernel<DT, D, 8>, (const void *)combine_kernel<DT, D, kWideRows>, Narrow<DT, D, 1>::SHARED, 8};
    return {(const void *)narrow_kernel<DT, D, 2>, (const void *)combine_kernel<DT, D, 16>, (const void *)combine_kernel<DT, D, kWideRows>, Narrow<DT, D, 2>::SHARED, 16};
}
template <int DT> static Kernels kernels_dt(int dim, int nt) {
    switch (dim) {
    case 32: return kernels_of<DT, 32>(nt);
    case 64: return kernels_of<DT, 64>(nt);
    case 96: return kernels_of<DT, 96>(nt);
    case 128: return kernels_of<DT, 128>(nt);
    case 192: return kernels_of<DT, 192>(nt);
    default: return kernels_of<DT, 256>(nt);
    }
}
// nt: eights of rows in a tile.
static Kernels kernels_for(const xgen_attention_desc &d, int nt) {
    return d.dtype == XGEN_F32 ? kernels_dt<XGEN_F32>(d.head_dim, nt) : kernels_dt<XGEN_F16_F32ACC>(d.head_dim, nt);
}
template <int ITEMS> static const void *append_of(xgen_dtype t) {
    return t == XGEN_F32 ? (const void *)append_kernel<XGEN_F32, ITEMS> : (const void *)append_kernel<XGEN_F16_F32ACC, ITEMS>;
}
static const void *append_for(xgen_dtype t, int items) { return items == 2 ? append_of<2>(t) : append_of<4>(t); }
static const void *read_for(xgen_dtype t) { return t == XGEN_F32 ? (const void *)read_kernel<XGEN_F32> : (const void *)read_kernel<XGEN_F16_F32ACC>; }

// ---- checks ----------------------------------------------------------------------------------------------------------------------
static xgen_status check_batch(const xgen_attention_batch *b, bool pointers) {
    if (!b) return XGEN_ERR_INVALID_ARG;
    if (b->sequences < 0 || b->sequences == INT32_MAX || b->rows < 0 || b->rows > INT32_MAX || b->longest < 0 || b->table_stride < 0 || b->table_stride > INT32_MAX)
        return XGEN_ERR_SHAPE;
    if (!pointers || b->sequences == 0 || b->rows == 0) return XGEN_OK;
    if (b->longest < 1 || b->table_stride < 1) return XGEN_ERR_SHAPE;
    if (!b->row_start_dev || !b->length_dev || !b->page_table_dev ||
        ((uintptr_t)b->row_start_dev | (uintptr_t)b->length_dev | (uintptr_t)b->page_table_dev) % 4)
        return XGEN_ERR_INVALID_ARG;
    return XGEN_OK;
}
static xgen_status check_cache(const xgen_attention_cache *c) {
    if (!c || !c->k_codes_dev || !c->v_codes_dev || !c->k_scale_dev || !c->v_scale_dev) return XGEN_ERR_INVALID_ARG;
    if (((uintptr_t)c->k_codes_dev | (uintptr_t)c->v_codes_dev) % 16 || ((uintptr_t)c->k_scale_dev | (uintptr_t)c->v_scale_dev) % 4) return XGEN_ERR_INVALID_ARG;
    if (c->pages < 1 || c->pages > INT32_MAX) return XGEN_ERR_SHAPE;
    return XGEN_OK;
}
static Batch batch_of(const xgen_attention_batch &b) {
    return {b.row_start_dev, b.length_dev, b.page_table_dev, b.table_stride, b.sequences, (int)b.rows, b.longest};
}
static Cache cache_of(const xgen_attention_packed &h, const xgen_attention_cache &c) {
    return {{static_cast<int8_t *>(c.k_codes_dev), static_cast<int8_t *>(c.v_codes_dev)}, {c.k_scale_dev, c.v_scale_dev}, c.pages, h.d.kv_heads, h.d.page_tokens, __builtin_ctz(h.d.page_tokens)};
}
static Rotation rotation_of(const xgen_attention_packed &h) { return {h.d_freq, reinterpret_cast<const float2 *>(h.d_freq + h.d.rotary / 2), h.d.rotary, h.d.interleaved}; }
static size_t span_bytes(int64_t rows, int64_t stride, int64_t width, size_t eb) { return ((size_t)(rows - 1) * stride + width) * eb; }
// Whether the bytes meet any of the cache's.
static bool in_cache(const xgen_attention_packed &h, const xgen_attention_cache &c, const void *p, size_t n) {
    const size_t scales = (size_t)c.pages * h.d.kv_heads * 4, codes = (size_t)c.pages * h.d.kv_heads * h.d.page_tokens * h.d.head_dim;
    return overlap(p, n, c.k_codes_dev, codes) || overlap(p, n, c.v_codes_dev, codes) || overlap(p, n, c.k_scale_dev, scales) || overlap(p, n, c.v_scale_dev, scales);
}
// Whether the bytes meet what describes the batch.
static bool in_batch(const xgen_attention_batch &b, const void *p, size_t n) {
    const size_t s = (size_t)b.sequences;
    return overlap(p, n, b.row_start_dev, (s + 1) * 4) || overlap(p, n, b.length_dev, s * 4) || overlap(p, n, b.page_table_dev, s * (size_t)b.table_stride * 4);
}
// Whether the parts of a cache meet each other, or the batch.
static bool cache_is_apart(const xgen_attention_packed &h, const xgen_attention_batch &b, const xgen_attention_cache &c) {
    const size_t scales = (size_t)c.pages * h.d.kv_heads * 4, codes = (size_t)c.pages * h.d.kv_heads * h.d.page_tokens * h.d.head_dim;
    const struct { const void *p; size_t n; } part[] = {{c.k_codes_dev, codes}, {c.v_codes_dev, codes}, {c.k_scale_dev, scales}, {c.v_scale_dev, scales}};
    for (int i = 0; i < 4; ++i) {
        if (in_batch(b, part[i].p, part[i].n)) return false;
        for (int o = 0; o < i; ++o)
            if (overlap(part[i].p, part[i].n, part[o].p, part[o].n)) return false;
    }
    return true;
}
// Whether two sets of rows of `width` bytes, `stride` apart in both, share a byte: those of one may lie between those of the other.
static bool rows_meet(const void *a, const void *b, int64_t rows, size_t stride, size_t width) {
    const size_t d = (uintptr_t)a < (uintptr_t)b ? (uintptr_t)b - (uintptr_t)a : (uintptr_t)a - (uintptr_t)b;
    const size_t n = d / stride, rest = d % stride;                    // row 0 of the later one begins in row n of the other, or behind it
    return (n < (size_t)rows && rest < width) || (n + 1 < (size_t)rows && stride - rest < width);
}
// Pages that the batch's rows reach, at most: n tokens of a sequence reach (n - 1)/page_tokens + 2 of them, and not more than n.
static int64_t pages_of(const xgen_attention_packed &h, const xgen_attention_batch &b) {
    const int64_t pages = b.rows / h.d.page_tokens + 2 * (int64_t)b.sequences;
    return pages < b.rows ? pages : b.rows;
}
// Heads of a block that takes a page's tokens: as many as leave eight blocks to an SM, so that what a block spends on finding its page counts
// little where there is much to do.  `sides`: 2 where keys and values go to blocks of their own.
static int heads_of_block(const xgen_attention_packed &h, int64_t pages, int sides) {
    int heads = 1;
    while (heads < h.d.kv_heads && pages * sides * ((h.d.kv_heads + heads) / (heads + 1)) >= 8 * (int64_t)h.sms) ++heads;
    return heads;
}
// Which kernels a call launches.
struct Route {
    int eights;                 // narrow_kernel's tiles, in eights of rows; 0: not launched
    bool wide;
};
// Few rows of every sequence (with all query heads of a key head) are narrow_kernel's, in tiles of eight where that holds them, else in tiles of
// 16.  Where a sequence may have more, wide_kernel takes those that have more than 16, and narrow_kernel is launched too unless
// all must have.  us by narrow_kernel and by wide_kernel, four query heads to a key head, dim 128, fp16: up to 32 rows of 8
// sequences over 8192 tokens 51 and 113, over 1024 28 and 72, of 64 over 2000 107 and 142; up to 64 rows 75 and 93, 30 and 47, and of 64
// sequences over 2000, where there are tiles enough for wide_kernel, 180 and 160: the rule looks at rows alone.  (Both, each with
// some of the sequences, are slower than either there: 115, 166, 61.)  More than kWideSequences sequences are narrow_kernel's, whatever their rows.
static Route route_of(const xgen_attention_packed &h, const xgen_attention_batch &b) {
    const int64_t group = h.d.q_heads / h.d.kv_heads, most = (int64_t)b.longest * group;
    if (most <= 8) return {1, false};
    if (most <= kNarrowAlone || !h.wide_workers || b.sequences > kWideSequences) return {2, false};
    const int64_t least = b.rows - (int64_t)(b.sequences - 1) * b.longest;       // rows of the shortest sequence, at least
    return {least * group > kNarrowMost ? 0 : 2, true};
}
static int64_t part_bytes(const xgen_attention_packed &h, int64_t workers, int64_t rows) {
    return (workers * 2 * rows * (h.d.head_dim * 4 + 16) + workers * (int64_t)sizeof(Cut) + 255) / 256 * 256;
}
static int64_t narrow_bytes(const xgen_attention_packed &h, const Route &r) { return r.eights ? part_bytes(h, h.workers[r.eights - 1], 8 * r.eights) : 0; }
static int64_t fold_bytes(const xgen_attention_packed &h) {
    return wide_kernel_for(h.d.dtype, h.d.head_dim).folds ? (int64_t)h.wide_workers * kWideRows * h.d.head_dim * 4 : 0;
}
// For any batch of at most these sequences, rows and rows of a sequence, whatever its route.
static int64_t workspace_of(const xgen_attention_packed &h, const xgen_attention_batch &b) {
    const int64_t most = (int64_t)b.longest * (h.d.q_heads / h.d.kv_heads), one = narrow_bytes(h, {1, false}), two = narrow_bytes(h, {2, false});
    if (most <= 8) return one;
    const int64_t narrow = one > two ? one : two;
    if (most <= kNarrowAlone || !h.wide_workers) return narrow;
    const int64_t rows = b.rows * h.d.q_heads, terms = wide_kernel_for(h.d.dtype, h.d.head_dim).terms;
    return narrow + part_bytes(h, h.wide_workers, kWideRows) + fold_bytes(h) + (rows * terms * h.d.head_dim + rows * 4 + 255) / 256 * 256;
}

}  // namespace attention

using namespace attention;

extern "C" {

xgen_status xgen_attention_pack(const xgen_attention_desc *d, const double *freq, int device, xgen_attention_packed **out) {
    if (!d || !out) return XGEN_ERR_INVALID_ARG;
    *out = nullptr;
    if (d->q_heads < 1 || d->kv_heads < 1 || d->q_heads % d->kv_heads || d->window < 0 || !(d->softmax_scale >= 0.0f) || !(d->softmax_scale < INFINITY) ||
        (d->rotary > 0) != (freq != nullptr))
        return XGEN_ERR_INVALID_ARG;
    if (d->dtype != XGEN_F32 && d->dtype != XGEN_F16_F32ACC) return XGEN_ERR_UNSUPPORTED;
    const int D = d->head_dim, pt = d->page_tokens;
    if ((D != 32 && D != 64 && D != 96 && D != 128 && D != 192 && D != 256) || (pt != 16 && pt != 32 && pt != 64 && pt != 128)) return XGEN_ERR_UNSUPPORTED;
    if (d->rotary < 0 || d->rotary > D || d->rotary % 2 || d->window > kLongest) return XGEN_ERR_UNSUPPORTED;
    if (d->q_heads > 65535) return XGEN_ERR_SHAPE;
    for (int u = 0; u < d->rotary / 2; ++u)
        if (!std::isfinite(freq[u])) return XGEN_ERR_INVALID_ARG;
    xgen_attention_packed *h = new (std::nothrow) xgen_attention_packed();
    if (!h) return XGEN_ERR_ALLOC;
    h->d = *d;
    h->d.interleaved = d->interleaved ? 1 : 0;
    if (h->d.softmax_scale == 0.0f) h->d.softmax_scale = (float)(1.0 / std::sqrt((double)D));
    h->device = device;
    if (device < 0) {
        *out = h;
        return XGEN_OK;
    }
    xgen_status st = XGEN_OK;
    OnDevice on(device);
    if (!on.ok) st = XGEN_ERR_CUDA;
    auto good = [&](cudaError_t e, xgen_status as) { if (st == XGEN_OK && e != cudaSuccess) st = as; };
    if (st == XGEN_OK) {
        good(cudaDeviceGetAttribute(&h->sms, cudaDevAttrMultiProcessorCount, device), XGEN_ERR_CUDA);
        for (int nt = 1; nt <= 2; ++nt) {
            const Kernels k = kernels_for(h->d, nt);
            int per_sm = 0;
            good(cudaFuncSetAttribute(k.narrow, cudaFuncAttributeMaxDynamicSharedMemorySize, k.shared), XGEN_ERR_CUDA);
            good(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, k.narrow, kThreads, k.shared), XGEN_ERR_CUDA);
            if (st == XGEN_OK && per_sm < 1) st = XGEN_ERR_CUDA;
            h->workers[nt - 1] = h->sms * per_sm;
        }
        const WideKernel wide = wide_kernel_for(h->d.dtype, h->d.head_dim);
        if (wide.kernel) {
            good(cudaFuncSetAttribute(wide.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, wide.shared), XGEN_ERR_CUDA);
            h->wide_workers = h->sms * wide.blocks;
        }
        good(cudaMalloc((void **)&h->d_status, 8), XGEN_ERR_ALLOC);
        if (st == XGEN_OK) good(cudaMemset(h->d_status, 0, 8), XGEN_ERR_CUDA);
    }
    if (st == XGEN_OK && d->rotary) {
        const int pairs = d->rotary / 2;
        std::vector<uint64_t> table;
        try {
            table.resize((size_t)pairs * (1 + h->d.page_tokens));
        } catch (const std::bad_alloc &) {
            st = XGEN_ERR_ALLOC;
        }
        for (int u = 0; u < pairs && st == XGEN_OK; ++u) {
            const long double whole = (long double)freq[u] / 6.283185307179586476925286766559005768L;
            const long double part = whole - floorl(whole);
            table[u] = (uint64_t)fminl(part * 18446744073709551616.0L, 18446744073709551615.0L);
            for (int slot = 0; slot < h->d.page_tokens; ++slot) {
                const long double turns = part * slot, at = (turns - floorl(turns)) * 6.283185307179586476925286766559005768L;
                const float cs[2] = {(float)cosl(at), (float)sinl(at)};
                std::memcpy(&table[pairs + (size_t)slot * pairs + u], cs, 8);
            }
        }
        if (st == XGEN_OK) good(cudaMalloc((void **)&h->d_freq, table.size() * 8), XGEN_ERR_ALLOC);
        if (st == XGEN_OK) good(cudaMemcpy(h->d_freq, table.data(), table.size() * 8, cudaMemcpyHostToDevice), XGEN_ERR_CUDA);
    }
    if (st == XGEN_OK) good(cudaDeviceSynchronize(), XGEN_ERR_CUDA);
    if (st != XGEN_OK) {
        cudaGetLastError();
        xgen_attention_free(h);
        return st;
    }
    *out = h;
    return XGEN_OK;
}

xgen_status xgen_attention_append(const xgen_attention_packed *h, const void *k, const void *v, int64_t stride, const xgen_attention_batch *b,
                                  const xgen_attention_cache *c, void *stream) {
    if (!h) return XGEN_ERR_INVALID_ARG;
    xgen_status st = check_batch(b, true);
    if (st == XGEN_OK) st = check_cache(c);
    if (st != XGEN_OK) return st;
    const int64_t width = (int64_t)h->d.kv_heads * h->d.head_dim;
    if (stride < width || stride > (1ll << 31)) return XGEN_ERR_SHAPE;
    if (b->sequences == 0 || b->rows == 0) return XGEN_OK;
    if (!k || !v) return XGEN_ERR_INVALID_ARG;
    const size_t eb = element_bytes(h->d.dtype), bytes = span_bytes(b->rows, stride, width, eb);
    if (((uintptr_t)k | (uintptr_t)v) % eb || in_cache(*h, *c, k, bytes) || in_cache(*h, *c, v, bytes) || !cache_is_apart(*h, *b, *c)) return XGEN_ERR_INVALID_ARG;
    if (h->device < 0) return XGEN_ERR_CUDA;
    AppendParams P{};
    P.batch = batch_of(*b); P.cache = cache_of(*h, *c); P.rotation = rotation_of(*h);
    P.in[0] = k; P.in[1] = v; P.stride = stride; P.dim = h->d.head_dim; P.status = h->d_status;
    for (int i = 0; i < 2; ++i) P.vec[i] = (uintptr_t)P.in[i] % 16 == 0 && stride * eb % 16 == 0;
    const int64_t pages = pages_of(*h, *b);
    OnDevice on(h->device);
    if (!on.ok) return XGEN_ERR_CUDA;
    void *args[] = {&P};
    const int tokens = h->d.page_tokens < b->longest ? h->d.page_tokens : b->longest;
    const int per_token = h->d.head_dim / 16, step = h->d.head_dim % 96 ? 32 : 96;        // threads: whole warps, and whole tokens
    // Two items a thread or four, us (with reading back) for 11.6 thousand rows, fp16: 8 heads of 128 in pages of 16 tokens 57 and 69, of 32
    // 51 and 58, of 64 54 and 47; heads of 64 in pages of 64 32 and 35, of 128 36 and 31.  64 rows: 10.4 and 11.1.  (Taken with codes by
    // the reciprocal alone, which saved 2 us of either.)
    const int items = tokens * per_token <= 256 ? 2 : 4;
    const int threads = (tokens * per_token + step * items - 1) / (step * items) * step;
    P.room = threads * items / per_token;
    P.heads = heads_of_block(*h, pages, 2);
    return launch(append_for(h->d.dtype, items), dim3((unsigned)pages, (h->d.kv_heads + P.heads - 1) / P.heads, 2), dim3(threads), 0, stream, args);
}

xgen_status xgen_attention_read(const xgen_attention_packed *h, const xgen_attention_batch *b, const xgen_attention_cache *c, xgen_dtype out_dtype,
                                void *k, void *v, int64_t stride, void *stream) {
    if (!h) return XGEN_ERR_INVALID_ARG;
    xgen_status st = check_batch(b, true);
    if (st == XGEN_OK) st = check_cache(c);
    if (st != XGEN_OK) return st;
    if (out_dtype != XGEN_F32 && out_dtype != XGEN_F16_F32ACC) return XGEN_ERR_UNSUPPORTED;
    const int64_t width = (int64_t)h->d.kv_heads * h->d.head_dim;
    if (stride < width || stride > (1ll << 31)) return XGEN_ERR_SHAPE;
    if (b->sequences == 0 || b->rows == 0) return XGEN_OK;
    if (!k || !v) return XGEN_ERR_INVALID_ARG;
    const size_t eb = element_bytes(out_dtype), bytes = span_bytes(b->rows, stride, width, eb);
    if (((uintptr_t)k | (uintptr_t)v) % eb || in_cache(*h, *c, k, bytes) || in_cache(*h, *c, v, bytes) || in_batch(*b, k, bytes) || in_batch(*b, v, bytes) ||
        rows_meet(k, v, b->rows, stride * eb, width * eb))
        return XGEN_ERR_INVALID_ARG;
    if (h->device < 0) return XGEN_ERR_CUDA;
    ReadParams P{};
    P.batch = batch_of(*b); P.cache = cache_of(*h, *c);
    P.out[0] = k; P.out[1] = v; P.stride = stride; P.dim = h->d.head_dim; P.status = h->d_status;
    const uint32_t per_token = (uint32_t)h->d.head_dim * (uint32_t)eb / 16;
    P.token_of = (uint32_t)(((1ull << 32) + per_token - 1) / per_token);   // (exact below 2^26 pieces: per_token is at most 64, a page has at most 2^13)
    for (int i = 0; i < 2; ++i) P.vec[i] = (uintptr_t)P.out[i] % 16 == 0 && stride * eb % 16 == 0;
    const int64_t pages = pages_of(*h, *b);
    P.heads = heads_of_block(*h, pages, 1);
    OnDevice on(h->device);
    if (!on.ok) return XGEN_ERR_CUDA;
    void *args[] = {&P};
    return launch(read_for(out_dtype), dim3((unsigned)pages, (h->d.kv_heads + P.heads - 1) / P.heads), dim3(kReadThreads), 0, stream, args);
}

xgen_status xgen_attention_workspace(const xgen_attention_packed *h, const xgen_attention_batch *b, int64_t *bytes) {
    if (!h || !bytes) return XGEN_ERR_INVALID_ARG;
    const xgen_status st = check_batch(b, false);
    if (st != XGEN_OK) return st;
    if (h->device < 0) return XGEN_ERR_CUDA;
    *bytes = workspace_of(*h, *b);
    return XGEN_OK;
}

xgen_status xgen_attention_run(const xgen_attention_packed *h, const void *q, int64_t q_stride, const xgen_attention_batch *b, const xgen_attention_cache *c,
                               void *y, int64_t y_stride, void *workspace, void *stream) {
    if (!h) return XGEN_ERR_INVALID_ARG;
    xgen_status st = check_batch(b, true);
    if (st == XGEN_OK) st = check_cache(c);
    if (st != XGEN_OK) return st;
    const int64_t width = (int64_t)h->d.q_heads * h->d.head_dim;
    const int group = h->d.q_heads / h->d.kv_heads;
    if (q_stride < width || y_stride < width || q_stride > (1ll << 31) || y_stride > (1ll << 31) || b->rows * group > INT32_MAX - 256) return XGEN_ERR_SHAPE;
    if (b->sequences == 0 || b->rows == 0) return XGEN_OK;
    if (!q || !y || !workspace) return XGEN_ERR_INVALID_ARG;
    const size_t eb = element_bytes(h->d.dtype), y_bytes = span_bytes(b->rows, y_stride, width, eb), q_bytes = span_bytes(b->rows, q_stride, width, eb);
    if (((uintptr_t)q | (uintptr_t)y) % eb || (uintptr_t)workspace % 16 || overlap(y, y_bytes, q, q_bytes) ||
        in_cache(*h, *c, y, y_bytes) || in_batch(*b, y, y_bytes))
        return XGEN_ERR_INVALID_ARG;
    if (h->device < 0) return XGEN_ERR_CUDA;
    const size_t work_bytes = (size_t)workspace_of(*h, *b);
    if (overlap(workspace, work_bytes, y, y_bytes) || overlap(workspace, work_bytes, q, q_bytes) || in_cache(*h, *c, workspace, work_bytes) ||
        in_batch(*b, workspace, work_bytes))
        return XGEN_ERR_INVALID_ARG;
    const Route route = route_of(*h, *b);
    RunParams P{};
    P.batch = batch_of(*b); P.cache = cache_of(*h, *c); P.rotation = rotation_of(*h);
    P.q = q; P.y = y; P.q_stride = q_stride; P.y_stride = y_stride;
    P.group = group; P.window = h->d.window;
    P.scale = (float)((double)h->d.softmax_scale * 1.4426950408889634);
    P.status = h->d_status; P.early = 16;
    P.extra = h->extra_arrivals; P.limit_us = h->extra_arrivals ? 50000u : 2000000u;
    P.vec_y = (uintptr_t)y % 16 == 0 && y_stride * eb % 16 == 0;
    P.launched = (route.eights ? 1 : 0) + (route.wide ? 1 : 0);
    OnDevice on(h->device);
    if (!on.ok) return XGEN_ERR_CUDA;
    // a kernel over tiles of `rows` rows, and the joining of what its workers leave in pieces
    const auto attend = [&](const void *kernel, const void *combine, int workers, int rows, int threads, int shared, char *work) {
        P.workers = workers;
        P.partial = reinterpret_cast<float *>(work);
        P.stats = reinterpret_cast<float4 *>(P.partial + (int64_t)workers * 2 * rows * h->d.head_dim);
        P.cut = reinterpret_cast<Cut *>(P.stats + (int64_t)workers * 2 * rows);
        void *args[] = {&P};
        xgen_status r = launch(kernel, dim3(workers), dim3(threads), shared, stream, args);
        if (r == XGEN_OK && workers > 1) r = launch(combine, dim3(workers - 1, (rows + kCombineRows - 1) / kCombineRows), dim3(kCombineThreads), 0, stream, args);
        return r;
    };
    const Kernels k = kernels_for(h->d, route.eights ? route.eights : 1);
    char *const work = static_cast<char *>(workspace);
    if (route.eights) st = attend(k.narrow, k.combine, h->workers[route.eights - 1], k.rows, kThreads, k.shared, work);
    if (st == XGEN_OK && route.wide) {
        const WideKernel w = wide_kernel_for(h->d.dtype, h->d.head_dim);
        char *const behind = work + narrow_bytes(*h, route) + part_bytes(*h, h->wide_workers, kWideRows);
        P.fold = reinterpret_cast<float4 *>(behind);
        P.q_bytes = reinterpret_cast<int8_t *>(behind + fold_bytes(*h));
        P.q_factor = reinterpret_cast<float *>(P.q_bytes + b->rows * h->d.q_heads * (int64_t)w.terms * h->d.head_dim);
        const int64_t warps = b->rows * ((h->d.q_heads + kQueryHeads - 1) / kQueryHeads);
        void *args[] = {&P};
        st = launch(w.queries, dim3((unsigned)((warps + kQueryThreads / 32 - 1) / (kQueryThreads / 32))), dim3(kQueryThreads), 0, stream, args);
        if (st == XGEN_OK) st = attend(w.kernel, k.combine_wide, h->wide_workers, kWideRows, kWideThreads, w.shared, work + narrow_bytes(*h, route));
    }
    return st;
}

xgen_status xgen_attention_last_status(const xgen_attention_packed *h, void *stream) {
    if (!h) return XGEN_ERR_INVALID_ARG;
    if (h->device < 0) return XGEN_ERR_CUDA;
    return take_status(h->device, h->d_status, 2, stream);
}

xgen_status xgen_attention_test_expect_arrivals(xgen_attention_packed *h, int32_t extra) {
    if (!h || extra < 0 || extra > 1000) return XGEN_ERR_INVALID_ARG;
    h->extra_arrivals = extra;
    return XGEN_OK;
}

void xgen_attention_free(xgen_attention_packed *h) {
    if (!h) return;
    if (h->device >= 0) {
        OnDevice on(h->device);
        if (on.ok) {
            cudaFree(h->d_freq); cudaFree(h->d_status);
        }
    }
    delete h;
}

}  // extern "C"
