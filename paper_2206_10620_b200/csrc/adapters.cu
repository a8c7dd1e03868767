// libpatconv: low-rank adapters of many requests beside a shared product, for sm_100a, and their C ABI.
//
// out[r] = y[r] + s_a B_a (A_a x[r]).  One kernel does both products: a cluster of eight blocks takes up to ROWS rows of one
// request.  Each block multiplies its eighth of the input features (the sums over features are joined through the blocks'
// shared memory), then each computes its eighth of the output channels.  So an adapter's matrices are read by eight SMs side by
// side even for a single row, nothing goes through memory in between, and there is one launch.
//
// The operands of the matrix instructions come straight from memory: which feature is which index of a product's sum is free as
// long as both operands agree, so a lane takes 16 contiguous bytes of a row of x and the same 16 bytes of the rows of A.
// Which channel is which column is free too: a lane's sums are 8 contiguous channels of its rows, so y and out move
// 16 bytes at a time.
//
// fp16: the inner sums are brought to fp16 with a power of two for each row, so that no magnitude is lost or overflows.  fp32:
// three products of tf32 parts (high x high, high x low, low x high): what is dropped is 2^-22 of a product.
#include <climits>
#include <cstring>
#include <new>
#include <vector>

#include "adapters.h"
#include "serve.cuh"

struct xgen_adapters_packed {
    xgen_adapters_desc d;
    int device;
    int rp, kp, np;             // rank, features and channels as stored: rounded up, the rest zeros
    void *d_a, *d_b;            // [adapters][rp][kp], [adapters][np][rp]
    float *d_scale;
    int *d_status;
};

namespace adapters {
using namespace serve;

constexpr int kCluster = 8, kThreads = 128, kWarps = 4;

struct Params {
    const void *x, *y, *a, *b;
    void *out;
    const int32_t *row_start, *adapter;
    const float *scale;
    int *status;
    int64_t x_stride, y_stride, out_stride;
    int rows, requests, k, kp, n, np, rank, adapters;
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

// d += the products of one block of features: lane 4g + t holds elements t*E .. t*E + E - 1 of the block (E = 16 bytes' worth) of
// rows g (x0) and g + 8 (x1) of one operand and of row g (w) of the other.
template <int DT> __device__ __forceinline__ void mma_block(float (&d)[4], const uint4 &x0, const uint4 &x1, const uint4 &w);
template <> __device__ __forceinline__ void mma_block<XGEN_F16_F32ACC>(float (&d)[4], const uint4 &x0, const uint4 &x1, const uint4 &w) {
    const uint32_t a[4] = {x0.x, x1.x, x0.y, x1.y}, b[4] = {x0.z, x1.z, x0.w, x1.w};
    mma16(d, a, w.x, w.y);
    mma16(d, b, w.z, w.w);
}
__device__ __forceinline__ void mma_split(float (&d)[4], const float (&x)[4], float w0, float w1) {
    uint32_t ah[4], al[4], bh[2], bl[2];
#pragma unroll
    for (int i = 0; i < 4; ++i) split_tf32(x[i], ah[i], al[i]);
    split_tf32(w0, bh[0], bl[0]);
    split_tf32(w1, bh[1], bl[1]);
    mma_tf32(d, al, bh[0], bh[1]);
    mma_tf32(d, ah, bl[0], bl[1]);
    mma_tf32(d, ah, bh[0], bh[1]);
}
template <> __device__ __forceinline__ void mma_block<XGEN_F32>(float (&d)[4], const uint4 &x0, const uint4 &x1, const uint4 &w) {
    const float a[4] = {__uint_as_float(x0.x), __uint_as_float(x1.x), __uint_as_float(x0.y), __uint_as_float(x1.y)};
    const float b[4] = {__uint_as_float(x0.z), __uint_as_float(x1.z), __uint_as_float(x0.w), __uint_as_float(x1.w)};
    mma_split(d, a, __uint_as_float(w.x), __uint_as_float(w.y));
    mma_split(d, b, __uint_as_float(w.z), __uint_as_float(w.w));
}

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ float far_load(const float *p, int rank) {
    uint32_t a;
    float v;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
    return v;
}

// DT: type.  RP: rank as stored.  ROWS: 16 (the warps divide a block's features and channels among them) or 64 (16 rows each).
template <int DT, int RP, int ROWS> __global__ void __launch_bounds__(kThreads) adapters_kernel(const Params P) {
    using T = typename Elem<DT>::T;
    constexpr int E = 16 / sizeof(T), BLOCK = 4 * E, NT = RP / 8;
    constexpr bool WIDE = ROWS == 64;
    __shared__ __align__(16) float part[64 * RP];        // [warp][16][RP]: this block's share of the inner sums
    __shared__ __align__(16) float total[WIDE ? 64 * RP / kCluster : 1];
    __shared__ float row_scale[ROWS];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const int rank = (int)(blockIdx.x % kCluster);
    let_next();
    wait_before();
    const Tile tile = find_tile<ROWS>(P, (int)(blockIdx.x / kCluster));
    if (tile.count == 0) return;                         // (the whole cluster alike)
    int who = P.adapter[tile.request];
    if (who >= P.adapters) {
        if (tid == 0) atomicExch(P.status, 1);
        who = -1;
    }
    const int row0 = WIDE ? warp * 16 : 0;               // of the tile, where this warp's 16 rows begin
    const T *const y = static_cast<const T *>(P.y) + (int64_t)tile.row * P.y_stride;
    T *const out = static_cast<T *>(P.out) + (int64_t)tile.row * P.out_stride;
    const int blocks_n = P.np / 32;

    if (who < 0) {                                       // (the same for the whole cluster)
        if (P.in_place) return;
        for (int64_t i = (int64_t)rank * kThreads + tid; i < (int64_t)tile.count * P.n; i += kCluster * kThreads) {
            const int64_t r = i / P.n, c = i % P.n;
            out[r * P.out_stride + c] = y[r * P.y_stride + c];
        }
        return;
    }

    // ---- inner sums: x [16 rows] times A^T [RP], this block's blocks of features
    float acc[NT][4];
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.0f;
    {
        const int nb = P.kp / BLOCK;
        const int lo = nb * rank / kCluster, hi = nb * (rank + 1) / kCluster;
        const bool in0 = row0 + g < tile.count, in1 = row0 + g + 8 < tile.count;
        const T *const x0 = static_cast<const T *>(P.x) + (int64_t)(tile.row + (in0 ? row0 + g : 0)) * P.x_stride;
        const T *const x1 = static_cast<const T *>(P.x) + (int64_t)(tile.row + (in1 ? row0 + g + 8 : 0)) * P.x_stride;
        const T *const w = static_cast<const T *>(P.a) + ((int64_t)who * RP + g) * P.kp;
        auto fetch = [&](const T *row, bool in, int at) {
            uint4 r = make_uint4(0, 0, 0, 0);
            if (in) {
                if (P.vec_x && at + E <= P.k) r = __ldg(reinterpret_cast<const uint4 *>(row + at));
                else {
                    T v[E];
#pragma unroll
                    for (int e = 0; e < E; ++e) v[e] = at + e < P.k ? row[at + e] : T(0.0f);
                    memcpy(&r, v, 16);
                }
            }
            return r;
        };
#pragma unroll 2
        for (int b = WIDE ? lo : lo + warp; b < hi; b += WIDE ? 1 : kWarps) {
            const int at = b * BLOCK + t * E;
            const uint4 u0 = fetch(x0, in0, at), u1 = fetch(x1, in1, at);
#pragma unroll
            for (int j = 0; j < NT; ++j) mma_block<DT>(acc[j], u0, u1, __ldg(reinterpret_cast<const uint4 *>(w + (int64_t)8 * j * P.kp + at)));
        }
    }
    {
        float *const mine = part + warp * 16 * RP;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            *reinterpret_cast<float2 *>(mine + g * RP + 8 * j + 2 * t) = make_float2(acc[j][0], acc[j][1]);
            *reinterpret_cast<float2 *>(mine + (g + 8) * RP + 8 * j + 2 * t) = make_float2(acc[j][2], acc[j][3]);
        }
    }
    __syncthreads();
    if (!WIDE) {                                         // the four warps' shares, into the first one's place
        for (int i = tid; i < 16 * RP; i += kThreads) part[i] = (part[i] + part[16 * RP + i]) + (part[32 * RP + i] + part[48 * RP + i]);
    }
    cluster_arrive();
    cluster_wait();
    // ---- the cluster's shares, into this block's own memory: the sums of all eight
    if (WIDE) {                                          // each block adds up an eighth, then all fetch the eighths
        constexpr int EIGHTH = 64 * RP / kCluster;
        for (int i = tid; i < EIGHTH; i += kThreads) {
            float v = 0.0f;
#pragma unroll
            for (int c = 0; c < kCluster; ++c) v += far_load(part + rank * EIGHTH + i, c);
            total[i] = (rank * EIGHTH + i) % RP < P.rank ? v : 0.0f;      // (padding times an infinity is no 0)
        }
        cluster_arrive();
        cluster_wait();
        for (int i = tid; i < 64 * RP; i += kThreads) part[i] = far_load(total + i % EIGHTH, i / EIGHTH);
        __syncthreads();
    } else {
        float *const sums = part + 16 * RP;              // (a place that nobody reads from afar)
        for (int i = tid; i < 16 * RP; i += kThreads) {
            float v = 0.0f;
#pragma unroll
            for (int c = 0; c < kCluster; ++c) v += far_load(part + i, c);
            sums[i] = i % RP < P.rank ? v : 0.0f;
        }
        __syncthreads();
    }
    cluster_arrive();                                    // (nobody's memory goes before all have read it: waited for at the end)
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
    const bool in0 = row0 + g < tile.count, in1 = row0 + g + 8 < tile.count;
    const float f0 = row_scale[row0 + g], f1 = row_scale[row0 + g + 8];
    const float *const h0 = h + (row0 + g) * RP, *const h1 = h + (row0 + g + 8) * RP;
    constexpr int STEPS = RP / BLOCK > 0 ? RP / BLOCK : 1;       // 16 bytes of a row of B at a time (8 where the rank is 16 in fp16)
    constexpr bool HALF = RP < BLOCK;
    uint4 u0[DT == XGEN_F32 ? 1 : STEPS], u1[DT == XGEN_F32 ? 1 : STEPS];
    if constexpr (DT != XGEN_F32) {
        constexpr int W = HALF ? 4 : 8;
#pragma unroll
        for (int st = 0; st < STEPS; ++st) {
            uint32_t p[2][4] = {};
#pragma unroll
            for (int e = 0; e < W / 2; ++e) {
                const int at = st * BLOCK + t * W + 2 * e;
                const __half2 v0 = __floats2half2_rn(h0[at] * f0, h0[at + 1] * f0), v1 = __floats2half2_rn(h1[at] * f1, h1[at + 1] * f1);
                memcpy(&p[0][e], &v0, 4);
                memcpy(&p[1][e], &v1, 4);
            }
            u0[st] = make_uint4(p[0][0], p[0][1], p[0][2], p[0][3]);
            u1[st] = make_uint4(p[1][0], p[1][1], p[1][2], p[1][3]);
        }
    }
    const T *const B = static_cast<const T *>(P.b) + (int64_t)who * P.np * RP;
    const float s0 = s / f0, s1 = s / f1;
    const int lo = (int)((int64_t)blocks_n * rank / kCluster), hi = (int)((int64_t)blocks_n * (rank + 1) / kCluster);
    for (int b = WIDE ? lo : lo + warp; b < hi; b += WIDE ? 1 : kWarps) {
        float d[4][4] = {};
        // column g of tile j is channel 8 (g/2) + 2 j + g%2 of the 32: a lane's sums are then channels 8t .. 8t + 7
        const T *const w = B + (int64_t)(b * 32 + 8 * (g >> 1) + (g & 1)) * RP;
#pragma unroll
        for (int st = 0; st < STEPS; ++st) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (DT == XGEN_F32) {
                    const uint4 v0 = *reinterpret_cast<const uint4 *>(h0 + st * BLOCK + t * E), v1 = *reinterpret_cast<const uint4 *>(h1 + st * BLOCK + t * E);
                    mma_block<DT>(d[j], v0, v1, __ldg(reinterpret_cast<const uint4 *>(w + 2 * j * RP + st * BLOCK + t * E)));
                } else if constexpr (HALF) {
                    const uint2 v = __ldg(reinterpret_cast<const uint2 *>(w + 2 * j * RP + t * 4));
                    const uint32_t a[4] = {u0[0].x, u1[0].x, u0[0].y, u1[0].y};
                    mma16(d[j], a, v.x, v.y);
                } else mma_block<DT>(d[j], u0[st], u1[st], __ldg(reinterpret_cast<const uint4 *>(w + 2 * j * RP + st * BLOCK + t * E)));
            }
        }
        const int c = b * 32 + 8 * t;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            if (!(r ? in1 : in0) || c >= P.n) continue;
            const int row = row0 + g + 8 * r;
            const T *const from = y + (int64_t)row * P.y_stride + c;
            T *const to = out + (int64_t)row * P.out_stride + c;
            const float by = r ? s1 : s0;
            if (P.vec_y && c + 8 <= P.n) {
                T v[8];
                uint4 raw[8 / E];
#pragma unroll
                for (int i = 0; i < 8 / E; ++i) raw[i] = reinterpret_cast<const uint4 *>(from)[i];
                memcpy(v, raw, sizeof v);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = narrow<T>(fmaf(by, d[i >> 1][2 * r + (i & 1)], widen(v[i])));
                memcpy(raw, v, sizeof v);
#pragma unroll
                for (int i = 0; i < 8 / E; ++i) reinterpret_cast<uint4 *>(to)[i] = raw[i];
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (c + i < P.n) to[i] = narrow<T>(fmaf(by, d[i >> 1][2 * r + (i & 1)], widen(from[i])));
            }
        }
    }
    __syncwarp();
    cluster_wait();
}

template <int DT> static const void *kernel(int rp, bool wide) {
    switch (rp) {
    case 16: return wide ? (const void *)adapters_kernel<DT, 16, 64> : (const void *)adapters_kernel<DT, 16, 16>;
    case 32: return wide ? (const void *)adapters_kernel<DT, 32, 64> : (const void *)adapters_kernel<DT, 32, 16>;
    case 64: return wide ? (const void *)adapters_kernel<DT, 64, 64> : (const void *)adapters_kernel<DT, 64, 16>;
    default: return wide ? (const void *)adapters_kernel<DT, 128, 64> : (const void *)adapters_kernel<DT, 128, 16>;
    }
}

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
    const size_t na = (size_t)d->adapters * rp * kp * eb, nb = (size_t)d->adapters * rp * np * eb;
    if (na + nb > (size_t)1 << 40) return XGEN_ERR_SHAPE;
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
    if (st == XGEN_OK) {
        good(cudaMemset(h->d_status, 0, 4));
        good(cudaMemcpy(h->d_scale, scale, (size_t)d->adapters * 4, cudaMemcpyHostToDevice));
        // one matrix at a time, its rows padded
        const auto upload = [&](void *to, const void *from, int rows, int cols, int rows_p, int cols_p) {
            const size_t one = (size_t)rows_p * cols_p * eb;
            std::vector<char> padded;
            try {
                padded.assign(one, 0);
            } catch (const std::bad_alloc &) {
                st = XGEN_ERR_ALLOC;
            }
            for (int i = 0; i < d->adapters && st == XGEN_OK; ++i) {
                for (int r = 0; r < rows; ++r)
                    std::memcpy(padded.data() + (size_t)r * cols_p * eb, static_cast<const char *>(from) + ((size_t)i * rows + r) * cols * eb, (size_t)cols * eb);
                good(cudaMemcpy(static_cast<char *>(to) + i * one, padded.data(), one, cudaMemcpyHostToDevice));
            }
        };
        upload(h->d_a, a, d->rank, d->k, rp, kp);
        upload(h->d_b, b, d->c_out, d->rank, np, rp);
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
    const bool wide = rows / requests >= 32;
    const int64_t tiles = rows / (wide ? 64 : 16) + (requests < rows ? requests : rows);
    if (tiles > INT32_MAX / kCluster) return XGEN_ERR_SHAPE;
    OnDevice on(h->device);
    if (!on.ok) return XGEN_ERR_CUDA;
    void *args[] = {&P};
    return launch(h->d.dtype == XGEN_F32 ? kernel<XGEN_F32>(h->rp, wide) : kernel<XGEN_F16_F32ACC>(h->rp, wide), dim3((unsigned)(tiles * kCluster)),
                  dim3(kThreads), 0, stream, args, kCluster);
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
