// libpatconv: low-rank adapters of many requests beside a shared product, for sm_100a, and their C ABI.
//
// out[r] = y[r] + s_a B_a (A_a x[r]).  One kernel does both products: a cluster of eight blocks (four or two where there are many
// clusters) takes up to ROWS rows of one request.  Each block multiplies its part of the input features (the sums over features are
// joined through the blocks' shared memory), then each computes its part of the output channels.  So an adapter's matrices are read
// by eight SMs side by side even for a single row, nothing goes through memory in between, and there is one launch.
//
// Which feature is which index of a product's sum is free as long as both operands agree, so a lane takes 16 contiguous bytes of a
// row of x, and the matrices are stored as the lanes take them.  Which channel is which column is free too: a lane's sums are 8
// contiguous channels of its rows, so y and out move 16 bytes at a time.
//
// Few rows are bound by latency: a chain of a load, a product, two meetings of the cluster, a load, a product.  48 rows of 48
// requests, 4096 features and channels, rank 16, fp16: 9.2 us (7.6 MB, 1.2 us at the memory's rate); one row 6.2 us.  Many rows
// overlap the chains of the blocks on an SM: 4 requests of 4600 rows in all, the same sizes: rank 16 31 us, rank 64 45 us (18 us
// for the bytes), rank 128 52 us.  With the adapters' operands in registers instead of shared memory these were 39, 55 and 90 us; with
// clusters of eight 33, 53 and 85 us.  fp32, rank 64: 184 us, bound by the instructions that split numbers into tf32 parts (three
// products each: 28 TFLOP/s).
//
// fp16: the inner sums are brought to fp16 with a power of two for each row, so that no magnitude is lost or overflows.  fp32:
// three products of tf32 parts (high x high, high x low, low x high): what is dropped is 2^-21 of a product at most.
#include <climits>
#include <cstring>
#include <new>
#include <vector>

#include "adapters.h"
#include "ptx.cuh"
#include "serve.cuh"

struct xgen_adapters_packed {
    xgen_adapters_desc d;
    int device;
    int processors;
    int rp, kp, np;             // rank, features and channels as stored: rounded up, the rest zeros
    void *d_a, *d_b;            // [adapters][kp / block][rp][block], [adapters][np / 32][rp / block][4][32 lanes][16 bytes]: see Order
    float *d_scale;
    int *d_status;
};

namespace adapters {
using namespace serve;
using patconv::copy16;
using patconv::copy_commit;
using patconv::copy_wait;
using patconv::smem_u32;

constexpr int kCluster = 8;                              // the most blocks of a cluster

struct Params {
    const void *x, *y, *a, *b;
    void *out;
    const int32_t *row_start, *adapter;
    const float *scale;
    int *status;
    int64_t x_stride, y_stride, out_stride;
    int rows, requests, k, kp, n, np, rank, adapters, cluster;
    bool vec_x, vec_y, in_place;
};

// The rows of tile `want`: {first row, number of rows, request}, or number 0 when there are fewer tiles.  Every lane of the warp takes part.
struct Tile { int row, count, request; };
template <int ROWS> __device__ __forceinline__ Tile find_tile(const Params &P, int want) {
    const int lane = threadIdx.x & 31;
    int before = 0;
    for (int i0 = 0; i0 < P.requests; i0 += 32) {
        const int i = i0 + lane;
        int lo = 0, n = 0;
        if (i < P.requests) {
            lo = min(max(P.row_start[i], 0), P.rows);
            n = max(min(P.row_start[i + 1], P.rows) - lo, 0);
            if (P.in_place && P.adapter[i] < 0) n = 0;
        }
        const int tiles = (n + ROWS - 1) / ROWS;
        int upto = tiles;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int v = __shfl_up_sync(~0u, upto, d);
            if (lane >= d) upto += v;
        }
        const unsigned hit = __ballot_sync(~0u, want < before + upto);
        if (hit) {
            const int at = __ffs(hit) - 1;
            const int skipped = (want - before) - (__shfl_sync(~0u, upto, at) - __shfl_sync(~0u, tiles, at));
            const int row = __shfl_sync(~0u, lo, at) + skipped * ROWS;
            return {row, min(ROWS, __shfl_sync(~0u, n, at) - skipped * ROWS), i0 + at};
        }
        before += __shfl_sync(~0u, upto, 31);
    }
    return {0, 0, 0};
}

// x as the sum of two tf32 numbers (and a rest of 2^-22 of it).
__device__ __forceinline__ void split_tf32(float x, uint32_t &hi, uint32_t &lo) {
    asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(hi) : "f"(x));
    float rest = x - __uint_as_float(hi);
    if (!(fabsf(rest) < INFINITY)) {                 // infinities and NaN have no rest; the largest numbers must not round up
        rest = 0.0f;
        if (fabsf(x) < INFINITY) { hi = __float_as_uint(x) & 0xFFFFE000u; rest = x - __uint_as_float(hi); }
    }
    asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(lo) : "f"(rest));
}

// The same for several numbers at once, by cheap instructions where all are finite and not among the very largest: then no rest is
// infinite or NaN.  (A rest has 12 bits beside its sign; the last one is lost where it has them all, 2^-23 of x at most.)
template <int N> __device__ __forceinline__ void split_tf32(const float (&x)[N], uint32_t (&hi)[N], uint32_t (&lo)[N]) {
    float check = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        hi[i] = (__float_as_uint(x[i]) + 0x1000u) & 0xFFFFE000u;
        const float rest = x[i] - __uint_as_float(hi[i]);
        lo[i] = __float_as_uint(rest) & 0xFFFFE000u;
        check += rest;
    }
    if (__any_sync(~0u, !(fabsf(check) < INFINITY))) {
#pragma unroll
        for (int i = 0; i < N; ++i) split_tf32(x[i], hi[i], lo[i]);
    }
}

// The left operand of one block of features: lane 4g + t holds elements t*E .. t*E + E - 1 of the block (E = 16 bytes' worth) of
// rows g (x0) and g + 8 (x1); mma_block adds its products with row g of the right one (w) to d.
template <int DT> struct Left {
    uint32_t a[4], b[4];
    __device__ __forceinline__ Left(const uint4 &x0, const uint4 &x1) : a{x0.x, x1.x, x0.y, x1.y}, b{x0.z, x1.z, x0.w, x1.w} {}
};
template <> struct Left<XGEN_F32> {
    uint32_t hi[8], lo[8];
    __device__ __forceinline__ Left(const uint4 &x0, const uint4 &x1) {
        const float x[8] = {__uint_as_float(x0.x), __uint_as_float(x1.x), __uint_as_float(x0.y), __uint_as_float(x1.y),
                            __uint_as_float(x0.z), __uint_as_float(x1.z), __uint_as_float(x0.w), __uint_as_float(x1.w)};
        split_tf32(x, hi, lo);
    }
};
__device__ __forceinline__ void mma_block(float (&d)[4], const Left<XGEN_F16_F32ACC> &x, const uint4 &w) {
    mma16(d, x.a, w.x, w.y);
    mma16(d, x.b, w.z, w.w);
}
// (The matrix unit rounds sums toward zero: a block's products are added up apart, the large ones last, and the blocks' sums with rounding.
// As one sum over 4096 features they were off by 7.5e-6, root mean square.)
__device__ __forceinline__ void mma_block(float (&d)[4], const Left<XGEN_F32> &x, const uint4 &w) {
    const float v[4] = {__uint_as_float(w.x), __uint_as_float(w.y), __uint_as_float(w.z), __uint_as_float(w.w)};
    uint32_t hi[4], lo[4], ah[2][4], al[2][4];
    split_tf32(v, hi, lo);
    float block[4] = {};
#pragma unroll
    for (int i = 0; i < 8; ++i) { ah[i / 4][i % 4] = x.hi[i]; al[i / 4][i % 4] = x.lo[i]; }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        mma_tf32(block, al[i], hi[2 * i], hi[2 * i + 1]);
        mma_tf32(block, ah[i], lo[2 * i], lo[2 * i + 1]);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) mma_tf32(block, ah[i], hi[2 * i], hi[2 * i + 1]);
#pragma unroll
    for (int i = 0; i < 4; ++i) d[i] += block[i];
}

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ float4 far_load(const float *p, int rank) {
    uint32_t a;
    float4 v;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a) : "memory");
    return v;
}

__device__ __forceinline__ float4 operator+(const float4 &a, const float4 &b) { return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w); }

// How the matrices are stored: in the order in which the lanes of a warp take them, 16 bytes each, so that a load of a warp is one
// piece of 512 bytes.  (Strided rows, 64 bytes of each, take the L1 twice as long: 4600 rows at rank 128 took 162 us, 133 in this order.)
template <int DT, int RP> struct Order {
    static constexpr int E = DT == XGEN_F32 ? 4 : 8, BLOCK = 4 * E;
    static constexpr bool HALF = RP < BLOCK;                            // (rank 16 in fp16: a lane's 16 bytes are 8 of each of two columns)
    static constexpr int STEPS = HALF ? 1 : RP / BLOCK, LOADS = HALF ? 2 : 4;
};

// Many rows: the four warps of a group (64 rows) share the operands of an adapter; a step of theirs is a block of features (the inner
// sums) or of 32 channels (the outer product).  DEPTH steps lie in shared memory: the adapter's part, then each warp's own rows.
template <int DT, int RP> struct Ring {
    using O = Order<DT, RP>;
    static constexpr int DEPTH = 3, PIECES = 16 / O::E;                 // a warp's rows: so many times 512 bytes
    static constexpr int SHARED = RP / 8 > O::STEPS * O::LOADS ? RP / 8 : O::STEPS * O::LOADS;
    static constexpr int SLOT = (SHARED + 4 * PIECES) * 32;             // x 16 bytes
    static constexpr int BYTES = 2 * DEPTH * SLOT * 16;
};
__device__ __forceinline__ void group_sync(int group) { asm volatile("bar.sync %0, 128;" ::"r"(group + 1) : "memory"); }

// Blocks that an SM holds at once: as many as can have the registers without spilling more than a few.
constexpr int resident(int dt, int rp, bool wide) {
    return dt == XGEN_F32 ? (rp <= 16 ? (wide ? 3 : 4) : rp <= 32 ? (wide ? 2 : 3) : wide ? (rp <= 64 ? 2 : 1) : rp <= 64 ? 3 : 2)
                          : wide ? (rp <= 32 ? 4 : rp <= 64 ? 3 : 2) : rp <= 16 ? 6 : rp <= 32 ? 5 : rp <= 64 ? 3 : 2;
}

// DT: type.  RP: rank as stored.  ROWS: 16 (four warps divide a block's features and channels among them) or 64 (two warps to 16
// rows divide theirs).
template <int DT, int RP, int ROWS> __global__ void __launch_bounds__(ROWS == 64 ? 256 : 128, resident(DT, RP, ROWS == 64)) adapters_kernel(const Params P) {
    using T = typename Elem<DT>::T;
    using O = Order<DT, RP>;
    constexpr int E = O::E, BLOCK = O::BLOCK, NT = RP / 8;
    constexpr bool WIDE = ROWS == 64, HALF = O::HALF;
    constexpr int kThreads = WIDE ? 256 : 128, GROUPS = ROWS / 16, SHARE = kThreads / 32 / GROUPS;  // SHARE: warps that have the same rows
    using R = Ring<DT, RP>;
    constexpr int DEPTH = R::DEPTH;
    // few rows: a block of an adapter's operands is asked for while the one before is multiplied, as far as registers go
    constexpr bool AHEAD_IN = !WIDE && NT <= 8, AHEAD_OUT = !WIDE && RP * (int)sizeof(T) <= 128;
    extern __shared__ uint4 ring_of_all[];
    __shared__ __align__(16) float part[64 * RP];        // [16 rows][RP] four times: this block's share of the inner sums
    __shared__ float row_scale[ROWS];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const int C = P.cluster, rank = (int)blockIdx.x % C;
    let_next();
    wait_before();
    const Tile tile = find_tile<ROWS>(P, (int)blockIdx.x / C);
    if (tile.count == 0) return;                         // (the whole cluster alike)
    int who = P.adapter[tile.request];
    if (who >= P.adapters) {
        if (tid == 0) atomicExch(P.status, 1);
        who = -1;
    }
    // of the tile, where this warp's rows begin; which of the warps with the same rows it is
    const int row0 = warp % GROUPS * 16, turn = warp / GROUPS;
    uint4 *const ring = ring_of_all + turn * DEPTH * R::SLOT + lane;
    const int own = (R::SHARED + warp % 4 * R::PIECES) * 32;               // in a slot: (each lane reads what it copied itself)
    const T *const y = static_cast<const T *>(P.y) + (int64_t)tile.row * P.y_stride;
    T *const out = static_cast<T *>(P.out) + (int64_t)tile.row * P.out_stride;
    const int blocks_n = P.np / 32;

    if (who < 0) {                                       // (the same for the whole cluster)
        if (P.in_place) return;
        const int first = (int)((int64_t)blocks_n * rank / C) * 32, last = min((int)((int64_t)blocks_n * (rank + 1) / C) * 32, P.n);
        for (int r = warp; r < tile.count; r += kThreads / 32) {
            const T *const from = y + r * P.y_stride;
            T *const to = out + r * P.out_stride;
#pragma unroll 4
            for (int c = first + lane * E; c < last; c += 32 * E) {
                if (P.vec_y && c + E <= last) *reinterpret_cast<uint4 *>(to + c) = *reinterpret_cast<const uint4 *>(from + c);
                else
                    for (int i = c; i < min(c + E, last); ++i) to[i] = from[i];
            }
        }
        return;
    }

    // ---- inner sums: x [rows] times A^T [RP], this block's blocks of features
    bool in[2];                                          // rows g and g + 8
#pragma unroll
    for (int i = 0; i < 2; ++i) in[i] = row0 + 8 * i + g < tile.count;
    float acc[NT][4] = {};
    {
        const int nb = P.kp / BLOCK;
        const int lo = nb * rank / C, hi = nb * (rank + 1) / C;
        const T *const x = static_cast<const T *>(P.x) + (int64_t)tile.row * P.x_stride;
        const uint4 *const w = reinterpret_cast<const uint4 *>(static_cast<const T *>(P.a) + (int64_t)who * RP * P.kp) + lane;
        const auto part_of_row = [&](int i, int at) {    // features at .. of row i, where they are not all there or not aligned
            const T *const row = x + (row0 + 8 * i + g) * P.x_stride;
            T v[E];
            uint4 all;
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = in[i] && at + e < P.k ? row[at + e] : T(0.0f);
            memcpy(&all, v, 16);
            return all;
        };
        const auto stage = [&](int b, int slot) {        // (many rows)
            const int at = b * BLOCK + t * E;
            uint4 *const to = ring + slot * R::SLOT;
            if (b < hi) {
#pragma unroll
                for (int j = 0; j < NT; j += 4)
                    if (j + warp % 4 < NT) copy16(smem_u32(to + (j + warp % 4) * 32), w + ((int64_t)b * NT + j + warp % 4) * 32, 16);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if (in[i] && P.vec_x && at + E <= P.k) copy16(smem_u32(to + own + i * 32), x + (row0 + 8 * i + g) * P.x_stride + at, 16);
                    else to[own + i * 32] = part_of_row(i, at);
                }
            }
            copy_commit();
        };
        struct { uint4 u[2], w[NT]; } now, next;
        const auto ask = [&](int b, auto &f) {
            const int at = b * BLOCK + t * E;
#pragma unroll
            for (int i = 0; i < 2; ++i)
                f.u[i] = in[i] && P.vec_x && at + E <= P.k ? *reinterpret_cast<const uint4 *>(x + (row0 + 8 * i + g) * P.x_stride + at) : part_of_row(i, at);
#pragma unroll
            for (int j = 0; j < NT; ++j) f.w[j] = __ldg(w + ((int64_t)b * NT + j) * 32);
        };
        if constexpr (WIDE) {
#pragma unroll
            for (int i = 0; i < DEPTH - 1; ++i) stage(lo + turn + i * SHARE, i);
            int slot = 0;
#pragma unroll 1
            for (int b = lo + turn; b < hi; b += SHARE) {
                copy_wait<DEPTH - 2>();
                group_sync(turn);                        // (this step's copies are there, nobody reads the last step's any more)
                stage(b + (DEPTH - 1) * SHARE, slot == 0 ? DEPTH - 1 : slot - 1);
                const uint4 *const from = ring + slot * R::SLOT;
                const Left<DT> left(from[own], from[own + 32]);
#pragma unroll
                for (int j = 0; j < NT; ++j) mma_block(acc[j], left, from[j * 32]);
                slot = slot + 1 == DEPTH ? 0 : slot + 1;
            }
            group_sync(turn);
        } else {
            int b = lo + turn;
            if (AHEAD_IN && b < hi) ask(b, now);
            for (; b < hi; b += SHARE) {
                if (!AHEAD_IN) ask(b, now);
                else if (b + SHARE < hi) ask(b + SHARE, next);
                const Left<DT> left(now.u[0], now.u[1]);
#pragma unroll
                for (int j = 0; j < NT; ++j) mma_block(acc[j], left, now.w[j]);
                if (AHEAD_IN) now = next;
            }
        }
    }
    // ---- what the outer product's first blocks of channels take is asked for ahead of the meetings
    const uint4 *const B = reinterpret_cast<const uint4 *>(static_cast<const T *>(P.b) + (int64_t)who * P.np * RP) + lane;
    const int out_lo = (int)((int64_t)blocks_n * rank / C), out_hi = (int)((int64_t)blocks_n * (rank + 1) / C);
    constexpr int STEPS = O::STEPS;
    struct Channels { uint4 w[STEPS][O::LOADS], y[2][8 / E]; };
    const auto ask = [&](int b, Channels &f) {
        // column g of tile j is channel 8 (g/2) + 2 j + g%2 of the 32: a lane's sums are then channels 8t .. 8t + 7
#pragma unroll
        for (int st = 0; st < STEPS; ++st)
#pragma unroll
            for (int j = 0; j < O::LOADS; ++j) f.w[st][j] = __ldg(B + (((int64_t)b * STEPS + st) * O::LOADS + j) * 32);
        const int c = b * 32 + 8 * t;
#pragma unroll
        for (int r = 0; r < 2; ++r)
            if (in[r] && P.vec_y && c + 8 <= P.n) {
#pragma unroll
                for (int i = 0; i < 8 / E; ++i) f.y[r][i] = reinterpret_cast<const uint4 *>(y + (int64_t)(row0 + g + 8 * r) * P.y_stride + c)[i];
            }
    };
    const auto stage = [&](int b, int slot) {            // (many rows)
        const int c = b * 32 + 8 * t;
        uint4 *const to = ring + slot * R::SLOT;
        if (b < out_hi) {
            constexpr int LOADS = STEPS * O::LOADS;
#pragma unroll
            for (int j = 0; j < LOADS; j += 4)
                if (j + warp % 4 < LOADS) copy16(smem_u32(to + (j + warp % 4) * 32), B + ((int64_t)b * LOADS + j + warp % 4) * 32, 16);
            if (P.vec_y && c + 8 <= P.n) {
#pragma unroll
                for (int r = 0; r < 2; ++r)
#pragma unroll
                    for (int i = 0; i < 8 / E; ++i)
                        if (in[r]) copy16(smem_u32(to + own + (r * (8 / E) + i) * 32), y + (int64_t)(row0 + g + 8 * r) * P.y_stride + c + i * E, 16);
            }
        }
        copy_commit();
    };
#pragma unroll
    for (int i = 0; i < (WIDE ? DEPTH - 1 : 0); ++i) stage(out_lo + turn + i * SHARE, i);
    Channels ahead;
    if (AHEAD_OUT && out_lo + turn < out_hi) ask(out_lo + turn, ahead);
    // ---- the shares of the warps with the same rows: side by side (16 rows), or each added to those before it
#pragma unroll
    for (int w = 0; w < (WIDE ? SHARE : 1); ++w) {
        if (!WIDE || turn == w) {
            float *const mine = part + (WIDE ? row0 : warp * 16) * RP;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    float2 &at = *reinterpret_cast<float2 *>(mine + (8 * i + g) * RP + 8 * j + 2 * t);
                    float2 v = make_float2(acc[j][2 * i], acc[j][2 * i + 1]);
                    if (w > 0) v = make_float2(at.x + v.x, at.y + v.y);
                    at = v;
                }
        }
        __syncthreads();
    }
    const auto keep = [&](int i, float4 v) {             // sums i .. i + 3 of all: a rank's padding times an infinity is no 0
        const int at = i % RP;
        return make_float4(at < P.rank ? v.x : 0.0f, at + 1 < P.rank ? v.y : 0.0f, at + 2 < P.rank ? v.z : 0.0f, at + 3 < P.rank ? v.w : 0.0f);
    };
    const auto four = [](float *p) -> float4 & { return *reinterpret_cast<float4 *>(p); };
    if (!WIDE) {                                         // the four warps' shares, into the first one's place
        for (int i = 4 * tid; i < 16 * RP; i += 4 * kThreads) four(part + i) = (four(part + i) + four(part + 16 * RP + i)) + (four(part + 32 * RP + i) + four(part + 48 * RP + i));
    }
    cluster_arrive();
    cluster_wait();
    // ---- the cluster's shares, into this block's own memory: the sums of all eight
    const auto all = [&](int i) {
        float4 v[kCluster] = {};
#pragma unroll
        for (int c = 0; c < kCluster; ++c)
            if (c < C) v[c] = far_load(part + i, c);
        return keep(i, ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7])));
    };
    // (nobody's memory goes before all have read it: waited for at the end)
    if (WIDE) {                                          // each block adds up its part of the sums, in place: nobody else reads that part here
        const int size = 64 * RP / C;
        for (int i = 4 * tid; i < size; i += 4 * kThreads) four(part + rank * size + i) = all(rank * size + i);
        cluster_arrive();
        cluster_wait();
#pragma unroll
        for (int i = 4 * tid; i < 64 * RP; i += 4 * kThreads)
            if (i / size != rank) four(part + i) = far_load(part + i, i / size);
    } else {                                             // (into a place that nobody reads from afar)
        for (int i = 4 * tid; i < 16 * RP; i += 4 * kThreads) four(part + 16 * RP + i) = all(i);
    }
    __syncthreads();
    cluster_arrive();
    const float *const h = WIDE ? part : part + 16 * RP;

    // ---- each row's power of two (fp16), with the adapter's scale
    for (int r = tid; r < ROWS; r += kThreads) {
        float most = 0.0f;
        for (int i = 0; i < RP; ++i) most = fmaxf(most, fabsf(h[r * RP + (i + r) % RP]));
        const int e = most > 0.0f && most < INFINITY ? min(max(exponent(most), -100), 126) : 0;
        row_scale[r] = DT == XGEN_F32 ? 1.0f : pow2(-e);
    }
    __syncthreads();
    const float s = P.scale[who];

    // ---- outer product: h [16 rows][RP] times B^T, 32 channels at a time
    constexpr int W = HALF ? 4 : E;                      // a lane's inner sums of a row at a time
    float by[2];
    uint4 u[2][STEPS];                               // (fp16)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int row = row0 + 8 * i + g;
        const float f = row_scale[row];
        by[i] = s / f;
        if constexpr (DT != XGEN_F32) {
#pragma unroll
            for (int st = 0; st < STEPS; ++st) {
                uint32_t p[4] = {};
#pragma unroll
                for (int e = 0; e < W / 2; ++e) {
                    const float2 two = *reinterpret_cast<const float2 *>(h + row * RP + st * BLOCK + t * W + 2 * e);
                    const __half2 v = __floats2half2_rn(two.x * f, two.y * f);
                    memcpy(&p[e], &v, 4);
                }
                u[i][st] = make_uint4(p[0], p[1], p[2], p[3]);
            }
        }
    }
    int slot = 0;
#pragma unroll 1
    for (int b = out_lo + turn; b < out_hi; b += SHARE) {
        Channels now;
        const uint4 *const from_ring = ring + slot * R::SLOT;
        if (WIDE) {
            copy_wait<DEPTH - 2>();
            group_sync(turn);
            stage(b + (DEPTH - 1) * SHARE, slot == 0 ? DEPTH - 1 : slot - 1);
            slot = slot + 1 == DEPTH ? 0 : slot + 1;
        } else if (AHEAD_OUT) {
            now = ahead;
            if (b + SHARE < out_hi) ask(b + SHARE, ahead);
        } else ask(b, now);
        const auto w = [&](int st, int j) { return WIDE ? from_ring[(st * O::LOADS + j) * 32] : now.w[st][j]; };
        const int c = b * 32 + 8 * t;
        float d[4][4] = {};
#pragma unroll
        for (int st = 0; st < STEPS; ++st) {
            if constexpr (HALF) {
                const uint32_t a[4] = {u[0][0].x, u[1][0].x, u[0][0].y, u[1][0].y};
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint4 v = w(0, j);
                    mma16(d[2 * j], a, v.x, v.y);
                    mma16(d[2 * j + 1], a, v.z, v.w);
                }
            } else {
                const auto of = [&](int i) { return DT == XGEN_F32 ? *reinterpret_cast<const uint4 *>(h + (row0 + 8 * i + g) * RP + st * BLOCK + t * E) : u[i][st]; };
                const Left<DT> left(of(0), of(1));
#pragma unroll
                for (int j = 0; j < 4; ++j) mma_block(d[j], left, w(st, j));
            }
        }
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            if (!in[r] || c >= P.n) continue;
            const int row = row0 + g + 8 * r;
            const T *const from = y + (int64_t)row * P.y_stride + c;
            T *const to = out + (int64_t)row * P.out_stride + c;
            const float f = by[r];
            if (P.vec_y && c + 8 <= P.n) {
                T v[8];
                uint4 raw[8 / E];
#pragma unroll
                for (int i = 0; i < 8 / E; ++i) memcpy(v + i * E, WIDE ? from_ring + own + (r * (8 / E) + i) * 32 : &now.y[r][i], 16);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = narrow<T>(fmaf(f, d[i >> 1][2 * r + (i & 1)], widen(v[i])));
                memcpy(raw, v, sizeof v);
#pragma unroll
                for (int i = 0; i < 8 / E; ++i) reinterpret_cast<uint4 *>(to)[i] = raw[i];
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (c + i < P.n) to[i] = narrow<T>(fmaf(f, d[i >> 1][2 * r + (i & 1)], widen(from[i])));
            }
        }
    }
    __syncwarp();
    cluster_wait();
}

constexpr int kSharedMost = 227 << 10;                   // of a block, with what the system keeps
constexpr int static_bytes(int rp) { return 256 * rp + 512; }
struct Kernel { const void *run; int shared; };
template <int DT, int RP> static Kernel kernel(bool wide) {
    return wide ? Kernel{(const void *)adapters_kernel<DT, RP, 64>, Ring<DT, RP>::BYTES} : Kernel{(const void *)adapters_kernel<DT, RP, 16>, 0};
}
template <int DT> static Kernel kernel(int rp, bool wide) {
    return rp == 16 ? kernel<DT, 16>(wide) : rp == 32 ? kernel<DT, 32>(wide) : rp == 64 ? kernel<DT, 64>(wide) : kernel<DT, 128>(wide);
}
static Kernel kernel_of(int dt, int rp, bool wide) { return dt == XGEN_F32 ? kernel<XGEN_F32>(rp, wide) : kernel<XGEN_F16_F32ACC>(rp, wide); }

}  // namespace adapters

using namespace adapters;

extern "C" {

xgen_status xgen_adapters_pack(const xgen_adapters_desc *d, const void *a, const void *b, const float *scale, int device,
                               xgen_adapters_packed **out) {
    if (!d || !a || !b || !scale || !out) return XGEN_ERR_INVALID_ARG;
    *out = nullptr;
    if (d->k < 1 || d->c_out < 1 || d->rank < 1 || d->adapters < 1) return XGEN_ERR_INVALID_ARG;
    if (d->rank > 128 || (d->dtype != XGEN_F32 && d->dtype != XGEN_F16_F32ACC)) return XGEN_ERR_UNSUPPORTED;
    if (d->k > 1 << 24 || d->c_out > 1 << 24) return XGEN_ERR_SHAPE;
    const size_t eb = element_bytes(d->dtype);
    const int rp = d->rank <= 16 ? 16 : d->rank <= 32 ? 32 : d->rank <= 64 ? 64 : 128;
    const int kp = (d->k + 31) / 32 * 32, np = (d->c_out + 31) / 32 * 32;
    const size_t one_a = (size_t)rp * kp * eb, one_b = (size_t)rp * np * eb;       // (2^33 at most)
    if ((size_t)d->adapters > ((size_t)1 << 40) / (one_a + one_b)) return XGEN_ERR_SHAPE;
    const size_t na = d->adapters * one_a, nb = d->adapters * one_b;
    xgen_adapters_packed *h = new (std::nothrow) xgen_adapters_packed();
    if (!h) return XGEN_ERR_ALLOC;
    h->d = *d; h->device = device; h->rp = rp; h->kp = kp; h->np = np;
    if (device < 0) {
        *out = h;
        return XGEN_OK;
    }
    xgen_status st = XGEN_OK;
    OnDevice on(device);
    if (!on.ok) st = XGEN_ERR_CUDA;
    auto alloc = [&](void **p, size_t n) {
        if (st == XGEN_OK && cudaMalloc(p, n) != cudaSuccess) st = XGEN_ERR_ALLOC;
    };
    alloc(&h->d_a, na);
    alloc(&h->d_b, nb);
    alloc((void **)&h->d_scale, (size_t)d->adapters * 4);
    alloc((void **)&h->d_status, 4);
    auto good = [&](cudaError_t e) { if (st == XGEN_OK && e != cudaSuccess) st = XGEN_ERR_CUDA; };
    for (int wide = 0; wide < 2 && st == XGEN_OK; ++wide)
        good(cudaFuncSetAttribute(kernel_of(d->dtype, rp, wide).run, cudaFuncAttributeMaxDynamicSharedMemorySize, kSharedMost - 1024 - static_bytes(rp)));
    if (st == XGEN_OK) {
        good(cudaDeviceGetAttribute(&h->processors, cudaDevAttrMultiProcessorCount, device));
        good(cudaMemset(h->d_status, 0, 4));
        good(cudaMemcpy(h->d_scale, scale, (size_t)d->adapters * 4, cudaMemcpyHostToDevice));
        // one matrix at a time, padded with zeros, in the order of struct Order; place(row, column): where an element goes, and
        // those behind it up to a multiple of `run` columns
        const auto upload = [&](void *to, const void *from, int rows, int cols, size_t elements, int run, auto place) {
            std::vector<char> stored;
            try {
                stored.assign(elements * eb, 0);
            } catch (const std::bad_alloc &) {
                st = XGEN_ERR_ALLOC;
            }
            for (int i = 0; i < d->adapters && st == XGEN_OK; ++i) {
                const char *at = static_cast<const char *>(from) + (size_t)i * rows * cols * eb;
                for (int r = 0; r < rows; ++r)
                    for (int c = 0; c < cols; c += run) {
                        const size_t n = (size_t)(cols - c < run ? cols - c : run) * eb;
                        std::memcpy(stored.data() + place(r, c) * eb, at, n);
                        at += n;
                    }
                good(cudaMemcpy(static_cast<char *>(to) + i * stored.size(), stored.data(), stored.size(), cudaMemcpyHostToDevice));
            }
        };
        const int e = (int)(16 / eb), block = 4 * e;
        upload(h->d_a, a, d->rank, d->k, (size_t)rp * kp, block, [&](int r, int f) { return ((size_t)(f / block) * rp + r) * block + f % block; });
        upload(h->d_b, b, d->c_out, d->rank, (size_t)rp * np, rp < block ? 4 : e, [&](int c, int r) {
            const bool half = rp < block;
            const int w = half ? 4 : e, j = c % 8 / 2, g = c % 32 / 8 * 2 + c % 2, lane = 4 * g + r / w % 4;
            const size_t step = (size_t)(c / 32) * (half ? 1 : rp / block) + r / (4 * w);
            return half ? ((step * 2 + j / 2) * 32 + lane) * 8 + j % 2 * 4 + r % w : ((step * 4 + j) * 32 + lane) * e + r % w;
        });
        good(cudaDeviceSynchronize());
    }
    if (st != XGEN_OK) {
        cudaGetLastError();
        xgen_adapters_free(h);
        return st;
    }
    *out = h;
    return XGEN_OK;
}

xgen_status xgen_adapters_run(const xgen_adapters_packed *h, const void *x, int64_t rows, int64_t x_stride, const int32_t *row_start,
                              const int32_t *adapter, int64_t requests, const void *y, int64_t y_stride, void *out, int64_t out_stride,
                              void *stream) {
    if (!h) return XGEN_ERR_INVALID_ARG;
    if (rows < 0 || requests < 0 || rows > INT32_MAX || requests > INT32_MAX - 1 || x_stride < h->d.k || y_stride < h->d.c_out ||
        out_stride < h->d.c_out || x_stride > (1ll << 31) || y_stride > (1ll << 31) || out_stride > (1ll << 31))
        return XGEN_ERR_SHAPE;
    if (rows == 0 || requests == 0) return XGEN_OK;
    if (!x || !row_start || !adapter || !y || !out) return XGEN_ERR_INVALID_ARG;
    const size_t eb = element_bytes(h->d.dtype);
    if (((uintptr_t)x | (uintptr_t)y | (uintptr_t)out) % eb || ((uintptr_t)row_start | (uintptr_t)adapter) % 4) return XGEN_ERR_INVALID_ARG;
    const bool in_place = y == out;
    const size_t out_bytes = ((size_t)(rows - 1) * out_stride + h->d.c_out) * eb;
    if (in_place ? y_stride != out_stride : overlap(out, out_bytes, y, ((size_t)(rows - 1) * y_stride + h->d.c_out) * eb)) return XGEN_ERR_INVALID_ARG;
    if (overlap(out, out_bytes, x, ((size_t)(rows - 1) * x_stride + h->d.k) * eb) || overlap(out, out_bytes, row_start, (size_t)(requests + 1) * 4) ||
        overlap(out, out_bytes, adapter, (size_t)requests * 4))
        return XGEN_ERR_INVALID_ARG;
    if (h->device < 0) return XGEN_ERR_CUDA;
    Params P{};
    P.x = x; P.y = y; P.out = out; P.a = h->d_a; P.b = h->d_b; P.scale = h->d_scale; P.status = h->d_status;
    P.row_start = row_start; P.adapter = adapter;
    P.x_stride = x_stride; P.y_stride = y_stride; P.out_stride = out_stride;
    P.rows = (int)rows; P.requests = (int)requests; P.k = h->d.k; P.kp = h->kp; P.n = h->d.c_out; P.np = h->np; P.rank = h->d.rank; P.adapters = h->d.adapters;
    P.vec_x = (uintptr_t)x % 16 == 0 && x_stride * eb % 16 == 0;
    P.vec_y = ((uintptr_t)y | (uintptr_t)out) % 16 == 0 && y_stride * eb % 16 == 0 && out_stride * eb % 16 == 0;
    P.in_place = in_place;
    // us by the kernel for many rows and by the other, rank 16, lengths from a third of the longest on: 64 requests of up to 96 rows 36 and
    // 50, of up to 144 53 and 40, of up to 300 69 and 79; 8 requests of up to 96 13.2 and 8.8, of 144 13.4 and 10.3, of 192 14.4 and 14.5;
    // 4 of up to 300 14.1 and 11.6, of 600 18 and 22, of 2048 32 and 44.  Below some 200 rows a request neither is the faster one throughout,
    // and an average says little of one long request among many short ones.
    const bool wide = rows / requests >= 64;
    const int64_t tiles = rows / (wide ? 64 : 16) + (requests < rows ? requests : rows);
    if (tiles > INT32_MAX / kCluster) return XGEN_ERR_SHAPE;
    // Clusters as large as all of them fit on the device at once: a few that come after the others take as long as those.
    // (Clusters of 8, 4, 2: 77 of many rows at rank 64 53, 46, 59 us, 317 of them 197, 162, 138 us; 200 single rows at rank 64 56,
    // 38, 32 us, 48 at rank 16 9.2, 10.2, 15.0 us.  At 1000 rows single blocks are 6 % faster still.)
    P.cluster = kCluster;
    while (P.cluster > 2 && tiles * P.cluster > h->processors * resident(h->d.dtype, h->rp, wide)) P.cluster /= 2;
    const Kernel k = kernel_of(h->d.dtype, h->rp, wide);
    // The device puts clusters side by side on an SM while others stay empty: memory that nobody uses keeps them apart.  (48 rows of 48
    // requests 11.0 us without, 9.2 with it; 4600 rows at rank 32 43.8 and 36.3 us.)  17/20: not every SM can be in a cluster.
    const int64_t need = (tiles * P.cluster * 20 + h->processors * 17 - 1) / (h->processors * 17);
    const int shared = max(k.shared, (int)(kSharedMost / need) - 1024 - static_bytes(h->rp));
    OnDevice on(h->device);
    if (!on.ok) return XGEN_ERR_CUDA;
    void *args[] = {&P};
    return launch(k.run, dim3((unsigned)(tiles * P.cluster)), dim3(wide ? 256 : 128), shared, stream, args, P.cluster);
}

xgen_status xgen_adapters_last_status(const xgen_adapters_packed *h, void *stream) {
    if (!h) return XGEN_ERR_INVALID_ARG;
    if (h->device < 0) return XGEN_ERR_CUDA;
    return take_status(h->device, h->d_status, 1, stream);
}

void xgen_adapters_free(xgen_adapters_packed *h) {
    if (!h) return;
    if (h->device >= 0) {
        OnDevice on(h->device);
        if (on.ok) {
            cudaFree(h->d_a); cudaFree(h->d_b); cudaFree(h->d_scale); cudaFree(h->d_status);
        }
    }
    delete h;
}

}  // extern "C"
