// libpatconv: log probabilities, entropy and top alternatives of rows of logits, for sm_100a, and their C ABI.
//
// One pass over the row: a thread takes every 512th 16-byte piece of its block's part and keeps the largest logit m so far,
// s = sum e^(x - m) and w = sum e^(x - m) (x - m); a larger logit rescales both.  Then lse = m + log s and the entropy is
// log s - w / s, with no difference of large numbers.  A row goes to a cluster of 1 to 16 blocks, so that a few rows fill
// the GPU too; the blocks' results meet in the first one's shared memory.
//
// The alternatives cost no second pass: `top` elements at least lie at or above the smallest of any `top` maxima of disjoint
// parts, so the top-th largest of the maxima of 32 parts (what lane i of any warp has seen) bounds the answer from below.
// Threads whose own maximum reaches it look through their pieces again (in L2 still) for what reaches it, on average some 30 to
// 130 elements for 32 parts, which are then ranked by comparing each with all.  Elements are compared as keys (logit, then
// lower index), so equal logits are no more trouble than others; where the order of the logits still leaves more than fit, the
// best element is taken out `top` times instead, the thread that had it looking for its next.
#include <math.h>

#include <climits>
#include <new>

#include "logprobs.h"
#include "serve.cuh"

struct xgen_logprobs_packed {
    xgen_logprobs_desc d;
    int device, sms;
};

namespace logprobs {
using namespace serve;

constexpr int kThreads = 512, kWarps = kThreads / 32, kTopMost = 32, kRoom = 1024;
constexpr float kLog2e = 1.4426950408889634f;

struct Params {
    const void *x;
    const int32_t *token;
    float *logprob, *entropy, *top_logprob;
    int32_t *top_index;
    int64_t stride;
    int vocab, top;
};

// Larger logits first, then lower indices: greater keys.
__device__ __forceinline__ uint32_t ordered(float v) {
    const uint32_t b = __float_as_uint(v == 0.0f ? 0.0f : v);            // -0 and 0 are equal
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }
__device__ __forceinline__ uint64_t key_of(float v, uint32_t index) { return (uint64_t)ordered(v) << 32 | (uint32_t)~index; }
constexpr uint64_t kNone = 0;                                             // below every key of a logit above -infinity

struct Sums { float m, s, w; };                 // the largest logit; sum e^(x-m); sum e^(x-m) (x-m)
__device__ __forceinline__ Sums joined(Sums a, Sums b) {
    const float m = fmaxf(a.m, b.m);
    const float da = a.m == m ? 0.0f : a.m - m, db = b.m == m ? 0.0f : b.m - m;       // (-inf and -inf: nothing on either side)
    const float ea = expf(da), eb = expf(db);
    Sums r;
    r.m = m;
    r.s = a.s * ea + b.s * eb;
    r.w = (ea > 0.0f ? (a.w + da * a.s) * ea : 0.0f) + (eb > 0.0f ? (b.w + db * b.s) * eb : 0.0f);
    return r;
}

template <int DT> struct Piece {       // 16 bytes of a row as one load
    using T = typename Elem<DT>::T;
    static constexpr int VEC = 16 / sizeof(T);
    float v[VEC];
    __device__ __forceinline__ void load(const T *p) {
        const uint4 r = __ldg(reinterpret_cast<const uint4 *>(p));
        if constexpr (DT == XGEN_F32) {
            v[0] = __uint_as_float(r.x); v[1] = __uint_as_float(r.y); v[2] = __uint_as_float(r.z); v[3] = __uint_as_float(r.w);
        } else {
            const uint32_t u[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&u[i]));
                v[2 * i] = f.x; v[2 * i + 1] = f.y;
            }
        }
    }
};

__device__ __forceinline__ uint32_t far_address(const void *p, int rank) {
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return a;
}
__device__ __forceinline__ void far_store(uint32_t a, float v) { asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(a), "f"(v) : "memory"); }
__device__ __forceinline__ void far_store(uint32_t a, uint64_t v) { asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(a), "l"(v) : "memory"); }

// DT: type of the logits.  The part of a row that a block owns: pieces [lo, hi) behind `head` single
// elements (up to the first 16-byte boundary), and the single elements behind the last piece; those at the ends belong to the
// first and the last block.
template <int DT> __global__ void __launch_bounds__(kThreads, 2) logprobs_kernel(const Params P, int cluster) {
    using T = typename Elem<DT>::T;
    constexpr int VEC = Piece<DT>::VEC;
    __shared__ Sums sums[kWarps];
    __shared__ uint64_t lane_top[kWarps][32];
    __shared__ uint64_t found[kRoom];
    __shared__ int n_found;
    __shared__ uint64_t best[kWarps];
    __shared__ uint64_t mine[kTopMost];
    __shared__ Sums far_sums[16];                                          // written by the cluster's blocks into the first one's
    __shared__ uint64_t far_top[16 * kTopMost];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int part = (int)(blockIdx.x % (unsigned)cluster);
    const int64_t row = blockIdx.x / (unsigned)cluster;
    if (cluster > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");       // every block has begun: waited for below
    wait_before();
    const T *const x = static_cast<const T *>(P.x) + row * P.stride;
    const int V = P.vocab;
    const int head = min(V, (int)(((16 - ((uintptr_t)x & 15)) & 15) / sizeof(T)));
    const int pieces = (V - head) / VEC;
    const int lo = (int)((int64_t)pieces * part / cluster), hi = (int)((int64_t)pieces * (part + 1) / cluster);
    const T *const body = x + head;
    // this thread's single elements: one of the head (threads 0..), one of the tail
    const int tail0 = head + pieces * VEC;
    const int one_head = part == 0 && tid < head ? tid : -1;
    const int one_tail = part == cluster - 1 && tid < V - tail0 ? tail0 + tid : -1;

    Sums a = {-INFINITY, 0.0f, 0.0f};
    int at_m = 0;                               // an index that the first element of that value does not lie behind
    float m2 = 0.0f;                            // m in powers of two as subtracted (rounded), or 0 while there is nothing
    auto raise = [&](float m, int last) {       // a new maximum, at index `last` or up to a piece before it
        at_m = last;
        if (DT == XGEN_F32) {
            const float d = a.m == -INFINITY ? 0.0f : a.m - m, e = expf(d);
            a.w = e > 0.0f ? (a.w + d * a.s) * e : 0.0f;
            a.s *= e;
        } else {
            const float n2 = m * kLog2e, d = m2 - n2, e = exp2_approx(a.s > 0.0f ? d : 0.0f);
            a.w = (a.w + d * a.s) * e;
            a.s *= e;
            m2 = n2;
        }
        a.m = m;
    };
    auto add = [&](float v) {
        if (DT == XGEN_F32) {                   // the difference first: a product of a large logit could overflow
            const float d = v - (a.m == -INFINITY ? 0.0f : a.m), e = exp2_approx(d * kLog2e);
            a.s += e;
            a.w += e * fmaxf(d, -200.0f);       // (e^-200 is 0: so -infinity adds 0, not a NaN)
        } else {
            const float d = fmaf(v, kLog2e, -m2), e = exp2_approx(d);
            a.s += e;
            a.w += e * fmaxf(d, -200.0f);
        }
    };
    auto single = [&](int i) {
        const float v = widen(x[i]);
        if (v > a.m) raise(v, i);
        add(v);
    };
    if (one_head >= 0) single(one_head);
    // pieces, four loads ahead
    constexpr int AHEAD = 4;
    auto take = [&](const Piece<DT> &p, int j) {
        float m = p.v[0];
#pragma unroll
        for (int i = 1; i < VEC; ++i) m = fmaxf(m, p.v[i]);
        if (m > a.m) raise(m, head + j * VEC + VEC - 1);
#pragma unroll
        for (int i = 0; i < VEC; ++i) add(p.v[i]);
    };
    int i = lo + tid;
    for (; i + (AHEAD - 1) * kThreads < hi; i += AHEAD * kThreads) {
        Piece<DT> p[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) p[u].load(body + (int64_t)(i + u * kThreads) * VEC);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) take(p[u], i + u * kThreads);
    }
    for (; i < hi; i += kThreads) {
        Piece<DT> p;
        p.load(body + (int64_t)i * VEC);
        take(p, i);
    }
    if (one_tail >= 0) single(one_tail);
    const float own_m = a.m;                    // this thread's largest logit (a NaN does not show here, but in s)
    if (DT != XGEN_F32 && a.m > -INFINITY) {    // from powers of two, relative to the rounded m2, to powers of e relative to m
        const float off = fmaf(-a.m, kLog2e, m2);
        a.w = (a.w + off * a.s) * 0.6931471805599453f;
        const float e = exp2_approx(off);
        a.s *= e; a.w *= e;
    }

    // ---- the block's sums, the maxima of its half warps
#pragma unroll
    for (int d = 16; d; d >>= 1) {
        const Sums b = {__shfl_xor_sync(~0u, a.m, d), __shfl_xor_sync(~0u, a.s, d), __shfl_xor_sync(~0u, a.w, d)};
        a = joined(a, b);
    }
    // (of the element that has this key or a greater one)
    const uint64_t own_key = own_m > -INFINITY ? key_of(own_m, (uint32_t)at_m) : kNone;
    if (lane == 0) sums[warp] = a;
    lane_top[warp][lane] = own_key;
    if (tid == 0) n_found = 0;
    __syncthreads();
    if (cluster > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    if (warp == 0) {
        Sums b = lane < kWarps ? sums[lane] : Sums{-INFINITY, 0.0f, 0.0f};
#pragma unroll
        for (int d = 16; d; d >>= 1) {
            const Sums c = {__shfl_xor_sync(~0u, b.m, d), __shfl_xor_sync(~0u, b.s, d), __shfl_xor_sync(~0u, b.w, d)};
            b = joined(b, c);
        }
        if (lane == 0) {
            if (cluster == 1) far_sums[0] = b;
            else {
                const uint32_t to = far_address(&far_sums[part], 0);
                far_store(to, b.m); far_store(to + 4, b.s); far_store(to + 8, b.w);
            }
        }
    }
    // ---- the block's alternatives, best first, in mine[]
    const int top = P.top;
    if (top > 0) {
        if (tid < kTopMost) mine[tid] = kNone;
        const uint64_t bound = [&] {            // the top-th largest of the 32 parts' keys (each warp works it out for itself)
            uint64_t v = lane_top[0][lane];
#pragma unroll
            for (int o = 1; o < kWarps; ++o) v = lane_top[o][lane] > v ? lane_top[o][lane] : v;
            int before = 0;
#pragma unroll
            for (int o = 0; o < 32; ++o) {
                const uint64_t u = __shfl_sync(~0u, v, o);
                before += u > v || (u == v && o < lane);
            }
            const unsigned at = __ballot_sync(~0u, before == top - 1);
            return __shfl_sync(~0u, v, __ffs(at) - 1);
        }();
        const float bound_value = bound == kNone ? -INFINITY : unordered((uint32_t)(bound >> 32));
        __syncthreads();
        auto look = [&](float v, int index) {
            if (v >= bound_value && v > -INFINITY) {
                const uint64_t k = key_of(v, (uint32_t)index);
                if (k < bound) return;
                const int at = atomicAdd(&n_found, 1);
                if (at < kRoom) found[at] = k;
            }
        };
        if (own_m >= bound_value && own_m > -INFINITY) {
            if (one_head >= 0) look(widen(x[one_head]), one_head);
#pragma unroll 4
            for (int j = lo + tid; j < hi; j += kThreads) {
                Piece<DT> p;
                p.load(body + (int64_t)j * VEC);
#pragma unroll
                for (int u = 0; u < VEC; ++u) look(p.v[u], head + j * VEC + u);
            }
            if (one_tail >= 0) look(widen(x[one_tail]), one_tail);
        }
        __syncthreads();
        const int n = n_found;
        if (n <= kRoom) {
            for (int c = tid; c < n; c += kThreads) {
                const uint64_t k = found[c];
                int rank = 0;
                for (int o = 0; o < n; ++o) rank += found[o] > k;
                if (rank < top) mine[rank] = k;
            }
        } else {
            // many equal logits: the best element `top` times over
            auto next_below = [&](uint64_t limit) {        // this thread's greatest key below limit
                uint64_t k = kNone;
                auto see = [&](float v, int index) {
                    const uint64_t c = key_of(v, (uint32_t)index);
                    if (v > -INFINITY && c < limit && c > k) k = c;
                };
                if (one_head >= 0) see(widen(x[one_head]), one_head);
                for (int j = lo + tid; j < hi; j += kThreads) {
                    Piece<DT> p;
                    p.load(body + (int64_t)j * VEC);
#pragma unroll
                    for (int u = 0; u < VEC; ++u) see(p.v[u], head + j * VEC + u);
                }
                if (one_tail >= 0) see(widen(x[one_tail]), one_tail);
                return k;
            };
            uint64_t k = next_below(~0ull);
            for (int r = 0; r < top; ++r) {
                uint64_t b = k;
#pragma unroll
                for (int d = 16; d; d >>= 1) {
                    const uint64_t o = __shfl_xor_sync(~0u, b, d);
                    b = o > b ? o : b;
                }
                if (lane == 0) best[warp] = b;
                __syncthreads();
                b = best[0];
                for (int o = 1; o < kWarps; ++o) b = best[o] > b ? best[o] : b;
                if (tid == 0) mine[r] = b;
                if (b != kNone && k == b) k = next_below(b);
                __syncthreads();
            }
        }
        __syncthreads();
        if (tid < top) {
            if (cluster == 1) far_top[tid] = mine[tid];
            else far_store(far_address(&far_top[part * kTopMost + tid], 0), mine[tid]);
        }
    }
    if (cluster > 1) {
        asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
        if (part) return;
    } else __syncthreads();

    // ---- the row's answers
    Sums r = far_sums[0];
    for (int c = 1; c < cluster; ++c) r = joined(r, far_sums[c]);
    const bool bad = isnan(r.s) || isnan(r.m) || r.m == INFINITY;
    const bool empty = !bad && r.m == -INFINITY;
    const float log_s = logf(r.s);
    auto answer = [&](float v) { return bad ? NAN : empty ? -INFINITY : (v - r.m) - log_s; };
    if (tid == 0 && P.logprob) {
        const int t = P.token[row];
        P.logprob[row] = t == -1 ? 0.0f : t < 0 || t >= V ? NAN : answer(widen(x[t]));
    }
    if (tid == 32 && P.entropy) P.entropy[row] = bad ? NAN : empty ? 0.0f : log_s - r.w / r.s;
    if (top > 0) {
        auto put = [&](int rank, uint64_t k) {
            P.top_index[row * top + rank] = bad || k == kNone ? -1 : (int)~(uint32_t)k;
            P.top_logprob[row * top + rank] = bad ? NAN : k == kNone ? -INFINITY : answer(unordered((uint32_t)(k >> 32)));
        };
        if (cluster == 1) {
            if (tid < top) put(tid, far_top[tid]);
        } else if (tid < cluster * kTopMost) {
            // an element's rank: its place in its own list, and how many of every other list are greater
            const int list = tid / kTopMost, at = tid % kTopMost;
            if (at < top) {
                const uint64_t k = far_top[list * kTopMost + at];
                int rank = at;
                for (int c = 0; c < cluster; ++c) {
                    if (c == list) continue;
                    int n = 0;                                   // entries of list c above k (empty ones: by list)
                    for (int step = 32; step; step >>= 1) {
                        const int probe = n + step - 1;
                        if (probe < top) {
                            const uint64_t o = far_top[c * kTopMost + probe];
                            if (o > k || (o == kNone && k == kNone && c < list)) n += step;
                        }
                    }
                    rank += n;
                }
                if (rank < top) put(rank, k);
            }
        }
    }
}

static const void *kernel_for(xgen_dtype t) {
    return t == XGEN_F32 ? (const void *)logprobs_kernel<XGEN_F32> : (const void *)logprobs_kernel<XGEN_F16_F32ACC>;
}

}  // namespace logprobs

using namespace logprobs;

extern "C" {

xgen_status xgen_logprobs_pack(const xgen_logprobs_desc *d, int device, xgen_logprobs_packed **out) {
    if (!d || !out) return XGEN_ERR_INVALID_ARG;
    *out = nullptr;
    if (d->vocab < 1 || d->top < 0 || d->top > kTopMost || d->top > d->vocab) return XGEN_ERR_INVALID_ARG;
    if (d->dtype != XGEN_F32 && d->dtype != XGEN_F16_F32ACC) return XGEN_ERR_UNSUPPORTED;
    int sms = 0;
    if (device >= 0 && cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess) {
        cudaGetLastError();
        return XGEN_ERR_CUDA;
    }
    xgen_logprobs_packed *h = new (std::nothrow) xgen_logprobs_packed();
    if (!h) return XGEN_ERR_ALLOC;
    h->d = *d; h->device = device; h->sms = sms;
    if (device >= 0) {          // clusters of 16 have to be asked for
        OnDevice on(device);
        if (!on.ok || cudaFuncSetAttribute(kernel_for(d->dtype), cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) {
            cudaGetLastError();
            delete h;
            return XGEN_ERR_CUDA;
        }
    }
    *out = h;
    return XGEN_OK;
}

xgen_status xgen_logprobs_run(const xgen_logprobs_packed *h, const void *x, int64_t rows, int64_t stride, const int32_t *token,
                              float *logprob, float *entropy, int32_t *top, float *top_logprob, void *stream) {
    if (!h) return XGEN_ERR_INVALID_ARG;
    if (rows < 0 || rows > INT32_MAX || stride < h->d.vocab || stride > (1ll << 31)) return XGEN_ERR_SHAPE;
    if ((logprob != nullptr) != (token != nullptr) || (top != nullptr) != (h->d.top > 0) || (top_logprob != nullptr) != (h->d.top > 0))
        return XGEN_ERR_INVALID_ARG;
    if (!logprob && !entropy && !top) return XGEN_ERR_INVALID_ARG;
    if (rows == 0) return XGEN_OK;
    if (!x) return XGEN_ERR_INVALID_ARG;
    const size_t eb = element_bytes(h->d.dtype);
    if ((uintptr_t)x % eb || ((uintptr_t)token | (uintptr_t)logprob | (uintptr_t)entropy | (uintptr_t)top | (uintptr_t)top_logprob) % 4)
        return XGEN_ERR_INVALID_ARG;
    {
        const struct { const void *p; size_t n; } all[] = {
            {x, ((size_t)(rows - 1) * stride + h->d.vocab) * eb}, {token, (size_t)rows * 4}, {logprob, (size_t)rows * 4},
            {entropy, (size_t)rows * 4}, {top, (size_t)rows * h->d.top * 4}, {top_logprob, (size_t)rows * h->d.top * 4}};
        for (int o = 2; o < 6; ++o)
            for (int i = 0; i < o; ++i)
                if (overlap(all[o].p, all[o].n, all[i].p, all[i].n)) return XGEN_ERR_INVALID_ARG;
    }
    if (h->device < 0) return XGEN_ERR_CUDA;
    Params P{};
    P.x = x; P.token = token; P.logprob = logprob; P.entropy = entropy; P.top_index = top; P.top_logprob = top_logprob;
    P.stride = stride; P.vocab = h->d.vocab; P.top = h->d.top;
    // Blocks to a row: as many as it takes to give every SM two, while a block's part is at least 8 KB.
    int cluster = 1;
    while (cluster < 16 && rows * cluster * 2 <= 2 * h->sms && (int64_t)P.vocab * (int64_t)eb / (cluster * 2) >= 8192) cluster *= 2;
    if (rows * cluster > INT32_MAX) return XGEN_ERR_SHAPE;
    OnDevice on(h->device);
    if (!on.ok) return XGEN_ERR_CUDA;
    void *args[] = {&P, &cluster};
    return launch(kernel_for(h->d.dtype), dim3((unsigned)(rows * cluster)),
                  dim3(kThreads), 0, stream, args, cluster);
}

void xgen_logprobs_free(xgen_logprobs_packed *h) { delete h; }

}  // extern "C"
