// What the attention kernels share: the batch and the cache as they see them, angles, codes, copies, integer products, the arguments of
// the kernels that attend.
#pragma once
#include <climits>
#include <cstring>

#include "attention.h"
#include "serve.cuh"

namespace attention {
using namespace serve;

// The batch and the cache as the kernels see them.
struct Batch {
    const int32_t *row_start, *length, *table;
    int64_t table_stride;
    int sequences, rows, longest;
};
struct Cache {
    int8_t *codes[2];           // keys, values
    float *scale[2];
    int64_t pages;
    int heads, page_tokens, page_shift;
};
struct Rotation {
    const uint64_t *freq;
    const float2 *slots;        // [page_tokens][rotary/2]: cosine and sine of slot times frequency
    int rotary, interleaved;
};

constexpr int kLongest = 1 << 30;    // tokens of a sequence
__device__ __forceinline__ int length_of(const Batch &B, int s) { return min(max(B.length[s], 0), kLongest); }
// First row and number of rows of a sequence.
struct Span { int row, n; };
__device__ __forceinline__ Span span_of(const Batch &B, int s) {
    const int lo = min(max(B.row_start[s], 0), B.rows);
    return {lo, max(min(B.row_start[s + 1], B.rows) - lo, 0)};
}
// The page of a token, or -1.
__device__ __forceinline__ int64_t page_of(const Batch &B, const Cache &C, int s, int token) {
    const int at = token >> C.page_shift;
    if (at >= B.table_stride) return -1;
    const int p = B.table[(int64_t)s * B.table_stride + at];
    return p >= 0 && p < C.pages ? p : -1;
}
// Components of pair u of a head of `dim`: those behind the turned ones pair up too, for convenience.
__device__ __forceinline__ int2 pair_of(const Rotation &R, int u) {
    if (u >= R.rotary / 2 || R.interleaved) return make_int2(2 * u, 2 * u + 1);
    return make_int2(u, u + R.rotary / 2);
}
// Cosine and sine of position times frequency.
__device__ __forceinline__ float2 angle(uint64_t freq, int position) {
    // in turns, modulo one turn: the upper half of a 64-bit product that wraps
    const int32_t frac = (int32_t)((freq * (uint64_t)position) >> 32);
    float2 r;
    sincospif((float)frac * 4.6566128730773926e-10f, &r.y, &r.x);    // 2^-31: half turns
    return r;
}
__device__ __forceinline__ void turn(float2 by, float &a, float &b) {
    const float x = a * by.x - b * by.y, y = a * by.y + b * by.x;
    a = x;
    b = y;
}

__device__ __forceinline__ float max_or_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float max_or_nan(float a, float b, float c) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// The sequence that a row belongs to, or ends before (the first one that ends behind it: 32 probes at a time); -1 behind the last.  Every
// lane of the warp takes part.
__device__ __forceinline__ int sequence_of_row(const Batch &B, int64_t row) {
    const int lane = threadIdx.x & 31;
    int lo = 0, hi = B.sequences;
    while (lo < hi) {
        const int step = (hi - lo + 31) / 32, probe = lo + lane * step;
        const unsigned behind = __ballot_sync(~0u, probe < hi && B.row_start[probe + 1] > row);
        const int first = behind ? __ffs(behind) - 1 : min(32, (hi - lo + step - 1) / step);       // probes before it end at or before the row
        if (behind) hi = min(hi, lo + first * step);
        if (first > 0) lo += (first - 1) * step + 1;
    }
    return lo < B.sequences ? lo : -1;
}
// Two of the four codes of `r` (its signs flipped: 0 .. 255) as fp16: 1024 + code as bits, less 1152.
template <int SELECT> __device__ __forceinline__ uint32_t widen_codes(uint32_t flipped) {
    const uint32_t b = __byte_perm(flipped, 0x64646464u, SELECT);
    const __half2 h = __hsub2(*reinterpret_cast<const __half2 *>(&b), __half2half2(__ushort_as_half(0x6480)));
    return *reinterpret_cast<const uint32_t *>(&h);
}

__device__ __forceinline__ uint32_t smem_at(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copy_async16(uint32_t to, const void *from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copy_async4(uint32_t to, const void *from) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copy_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void load_matrices(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void load_matrices_turned(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ uint32_t pack_half(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// D[16][8] += A[16][32] B[32][8] in signed bytes, 32-bit sums.  Lane 4g + t holds of A bytes 4t .. 4t + 3 of rows g (a[0]) and g + 8 (a[1]),
// and bytes 16 + 4t .. of both; of B rows 4t .. 4t + 3 of column g, and 16 + 4t ..; of D as in mma16.
__device__ __forceinline__ void mma_bytes(int (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// a / b for a >= 0, b > 0: mostly small enough for the short division.
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
    return (a | b) < (1ll << 32) ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}
// A row's sums are of probability times scale times code.  What goes into fp16 is the product of the first two, relative to the largest that
// the row has met so far, not the probability relative to the largest scale: a page of large values that hardly counts for the row, or that
// it does not see, must not cost the others their bits.  (Relative to the largest scale, a page 10^6 times smaller with all the weight kept
// 12 bits of the 22 in fp32 layers.)
// The row keeps, as whole numbers of powers of two, so that changing them rounds nothing, a reference m of its scores and one of its
// sums, `unit`, relative to m: sums are of p f 2^(e + kLift - unit) code for a scale f 2^e, p = 2^(score - m); -infinity: no sums yet.
// They go up where a score, or a product, lies more than 2^kFar above them.  So a product is at most 2^15 as it becomes fp16, which holds
// all its bits down to 2^-20 of the row's largest.  A probability of less than 2^-100 of the row's largest may count as none.
// (Scores are formed relative to m, in one rounding, so that far from 0 too they are no further above it than they are said to be.)
constexpr int kLift = 7;
constexpr float kFar = 7.0f;
// A scale as f times 2^e, 1 <= f < 2; e = -infinity for one that is not above 0, or not finite.
struct Split { float e, f; };
__device__ __forceinline__ Split split_scale(float v) {
    const bool least = v < 1.17549435e-38f;               // below the normal numbers
    const uint32_t u = __float_as_uint(least ? v * 4294967296.0f : v);
    if (!(v > 0.0f && v < INFINITY)) return {-INFINITY, 1.0f};
    return {(float)((int)(u >> 23) - (least ? 159 : 127)), __uint_as_float((u & 0x7FFFFFu) | 0x3F800000u)};
}
// The score reference once more where the largest score lies x above `base`; by how much it went up.  (Rounded up, where it has no room for units.)
__device__ __forceinline__ float raise_reference(float &m, float base, float x) {
    m = __fadd_ru(base, ceilf(x));
    return m - base;
}
// What a row's sums are to be multiplied by, one after the other (their product may not be a normal number): 2^(unit - kLift) / total.
__device__ __forceinline__ float2 result_factors(float total, float unit) {
    const float near = fminf(fmaxf(unit, -126.0f), 127.0f);
    return make_float2(total == 0.0f ? 0.0f : pow2(-kLift) / total * exp2_approx(unit - near), exp2_approx(near));
}

// Where a worker's piece of the line begins: the tile (its rows, the units that it takes, which unit of the line is its first), and the
// length of a piece.
struct __align__(16) Cut {
    int64_t first, piece;
    int units, row, n, head, row0, unused[3];       // units = 0: the worker has no piece
};
struct RunParams {
    Batch batch;
    Cache cache;
    Rotation rotation;
    const void *q;
    void *y;
    int64_t q_stride, y_stride;
    int group, window;
    bool vec_y;                      // rows of y start on multiples of 16 bytes
    float scale;                     // softmax scale times log2(e)
    float *partial;                  // [workers][2][rows of a tile][dim] sums
    float4 *stats;                   // [workers][2][rows of a tile]: reference m, total, unit of the sums
    struct Cut *cut;                 // [workers]
    int8_t *q_bytes;                 // wide_kernel: [kv_heads][rows * group][terms][dim]: the queries' integers, bytes of the lowest value first
    float *q_factor;                 // [kv_heads][rows * group]: what they are multiples of, times the scale
    float4 *fold;                    // wide_kernel: [workers][dim/4][128 rows], where a worker keeps totals that tensor memory has no room for
    int workers, early;
    uint32_t limit_us;               // of wide_kernel's waits
    int extra;                       // arrivals that its products' barrier waits for in vain (a testing aid)
    int launched;                    // how many kernels share the sequences: 1 (this one takes all) or 2
    int *status;
};


// Rows of a sequence (with all query heads of a key head) up to which narrow_kernel takes it where both kernels are launched.
constexpr int kNarrowMost = 16, kNarrowAlone = 64;      // beside wide_kernel; where there is none
// The kernel for many rows (attention_wide.cu): what one needs to launch it; no kernel where the block's memory would not do.
constexpr int kWideRows = 128, kWideThreads = kWideRows + 32, kWideUnit = 64, kWideSequences = 1024;
struct WideKernel {
    const void *kernel, *queries;    // `queries` goes before it
    int shared, blocks, terms;       // blocks: resident on an SM at once
    bool folds;                      // it takes RunParams::fold
};
constexpr int kQueryThreads = 256, kQueryHeads = 4;      // a warp of `queries` takes a row's kQueryHeads heads
WideKernel wide_kernel_for(xgen_dtype t, int dim);

}  // namespace attention
