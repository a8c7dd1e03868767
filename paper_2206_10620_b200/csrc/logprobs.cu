// libpatconv: log probabilities, entropy and top alternatives of rows of logits, for sm_100a, and their C ABI.
//
// One pass over the row: a thread takes every 256th 16-byte piece of its block's part and keeps a reference m near the largest logit
// so far (raised, and the sums rescaled, only where a logit lies 8 above it: e^8 is no strain on a sum), s = sum e^(x - m) and
// w = sum e^(x - m) (x - m).  Then lse = m + log s and the entropy is log s - w / s.  m may lie 8 below the largest logit, so where one
// token has nearly all of the probability these are differences of numbers of up to 8, off by some 1e-6, and held to their sign.  A row
// goes to a cluster of 1 to 16 blocks, so that a few rows fill the GPU too; what the blocks found meets in shared memory.
// (What follows the pass over the row is short code, loops not unrolled and sums joined by one function that is called: most of it is
// run once, and while the GPU reads its rows a line of instructions that no cache holds takes a microsecond to come.)
//
// The alternatives cost no second pass: `top` elements at least lie at or above the smallest of any `top` maxima of disjoint
// parts, so the top-th largest of the maxima of 32 parts (what lane i of any warp has seen) bounds the answer from below.
// Threads keep the maxima of up to 16 stretches of their pieces; the stretches whose maximum reaches the bound are looked through
// again (in L2 still) by all threads for what reaches it, on average some 30 to 130 elements of the whole row, which the first
// block then ranks by comparing each with all.  Elements are compared as keys (logit, then lower index), so equal logits are no more trouble than
// others; where the order of the logits still leaves more than fit, the best element is taken out `top` times instead, the
// thread that had it looking for its next.
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

constexpr int kThreads = 256, kWarps = kThreads / 32, kTopMost = 32, kRoom = 1024, kAhead = 2, kStages = 4, kStretches = 16;
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

struct Sums { float m, s, w; };                 // the reference; sum e^(x-m); sum e^(x-m) (x-m)
// The sums of several lanes of a warp in one (lanes without any hold m = -infinity, s = w = 0).
__device__ __noinline__ Sums joined(Sums a) {
    float m = a.m;
#pragma unroll 1
    for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, d));
    const float d = a.m == m ? 0.0f : a.m - m, e = exp2_approx(d * kLog2e);
    Sums r;
    r.m = m;
    r.w = e > 0.0f ? (a.w + d * a.s) * e : 0.0f;
    r.s = a.s * e;
#pragma unroll 1
    for (int o = 16; o; o >>= 1) {
        r.s += __shfl_xor_sync(~0u, r.s, o);
        r.w += __shfl_xor_sync(~0u, r.w, o);
    }
    return r;
}

// 16 bytes of a row.
template <int DT> struct Piece {
    using T = typename Elem<DT>::T;
    static constexpr int VEC = 16 / sizeof(T);
    uint32_t u[4];
    __device__ __forceinline__ void load(const T *p) {
        take(*reinterpret_cast<const uint4 *>(p));
    }
    __device__ __forceinline__ void take(const uint4 &r) {
        u[0] = r.x; u[1] = r.y; u[2] = r.z; u[3] = r.w;
    }
    __device__ __forceinline__ void nothing() {
        u[0] = u[1] = u[2] = u[3] = DT == XGEN_F32 ? 0xFF800000u : 0xFC00FC00u;
    }
    __device__ __forceinline__ float at(int i) const {
        if constexpr (DT == XGEN_F32) return __uint_as_float(u[i]);
        else {
            const __half2 h = *reinterpret_cast<const __half2 *>(&u[i >> 1]);
            return i & 1 ? __high2float(h) : __low2float(h);
        }
    }
    __device__ __forceinline__ float any(int i) const {     // at(), for a place known at run time
        const int w = DT == XGEN_F32 ? i : i >> 1;
        const uint32_t v = w < 2 ? (w == 0 ? u[0] : u[1]) : (w == 2 ? u[2] : u[3]);
        if constexpr (DT == XGEN_F32) return __uint_as_float(v);
        else return __half2float(__ushort_as_half((unsigned short)(v >> (16 * (i & 1)))));
    }
    __device__ __forceinline__ void one(T v) {              // that element, the others left as they are
        if constexpr (DT == XGEN_F32) u[0] = __float_as_uint(v);
        else u[0] = (u[0] & 0xFFFF0000u) | __half_as_ushort(v);
    }
    __device__ __forceinline__ float most() const {         // (leaves NaN out)
        if constexpr (DT == XGEN_F32)
            return fmaxf(fmaxf(__uint_as_float(u[0]), __uint_as_float(u[1])), fmaxf(__uint_as_float(u[2]), __uint_as_float(u[3])));
        else {
            const __half2 *const h = reinterpret_cast<const __half2 *>(u);
            const __half2 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
            return fmaxf(__low2float(m), __high2float(m));
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
__device__ __forceinline__ int far_load(uint32_t a) {
    int v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ int far_add(uint32_t a, int v) {
    int old;
    asm volatile("atom.shared::cluster.add.u32 %0, [%1], %2;" : "=r"(old) : "r"(a), "r"(v) : "memory");
    return old;
}
// The two halves of a meeting of the cluster's blocks (of the block's warps where it is alone).
__device__ __forceinline__ void arrive(int cluster) {
    if (cluster > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void await(int cluster) {
    if (cluster > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    else __syncthreads();
}

// The dynamic shared memory: pieces on their way, each thread's its own; once the row is read, what is found in it.
union Memory {
    uint4 ring[kStages][kAhead][kThreads];
    struct {
        uint64_t found[kRoom], lists[16 * kTopMost];
        uint16_t queue[kStretches * kThreads];              // stretches to be looked through: number * kThreads + thread
    } late;
};

// DT: type of the logits.  ENTROPY: whether it is asked for.  The part of a row that a block owns: pieces [lo, hi) behind `head` single
// elements (up to the first 16-byte boundary), and the single elements behind the last piece; those at the ends belong to the
// first and the last block.
template <int DT, bool ENTROPY> __global__ void __launch_bounds__(kThreads, 4) logprobs_kernel(const Params P, int cluster) {
    using T = typename Elem<DT>::T;
    constexpr int VEC = Piece<DT>::VEC;
    __shared__ Sums sums[kWarps];
    __shared__ uint64_t lane_top[kWarps][32];
    __shared__ uint64_t best[kWarps];
    __shared__ uint64_t bound_key;
    __shared__ float stretch_top[kStretches][kThreads];
    __shared__ int n_queue;
    // what the cluster's blocks write to each other: the 32 parts' keys to all; sums, what they found, their lists to the first
    __shared__ uint64_t far_lane_top[16][32];
    __shared__ Sums far_sums[16];
    __shared__ Sums all;
    __shared__ int n_found;
    extern __shared__ __align__(16) unsigned char dynamic[];
    Memory &mem = *reinterpret_cast<Memory *>(dynamic);
    uint64_t *const found = mem.late.found, *const lists = mem.late.lists;
    uint16_t *const queue = mem.late.queue;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int part = (int)(blockIdx.x % (unsigned)cluster);
    const int64_t row = blockIdx.x / (unsigned)cluster;
    if (tid == 0) n_found = n_queue = 0;
    arrive(cluster);                            // (every block has begun, its counter is set: waited for below)
    let_next();
    wait_before();
    const T *const x = static_cast<const T *>(P.x) + row * P.stride;
    const int V = P.vocab, top = P.top;
    int token = -1;
    float token_logit = 0.0f;
    if (tid == 0 && part == 0 && P.logprob) {
        token = P.token[row];
        if (token >= 0 && token < V) token_logit = widen(x[token]);
    }
    const int head = min(V, (int)(((16 - ((uintptr_t)x & 15)) & 15) / sizeof(T)));
    const int pieces = (V - head) / VEC;
    const int lo = (int)((int64_t)pieces * part / cluster), hi = (int)((int64_t)pieces * (part + 1) / cluster);
    const T *const body = x + head;
    // this thread's single elements: one of the head (threads 0..), one of the tail
    const int tail0 = head + pieces * VEC;
    const int one_head = part == 0 && tid < head ? tid : -1;
    const int one_tail = part == cluster - 1 && tid < V - tail0 ? tail0 + tid : -1;

    Sums a = {-INFINITY, 0.0f, 0.0f};
    float own_m = -INFINITY;                    // this thread's largest logit (a NaN does not show here, but in s)
    int at_m = 0;                               // an index that the first element of that value does not lie behind
    float m2 = 0.0f;                            // fp16: m in powers of two as subtracted (rounded); fp32: m; 0 while there is nothing
    constexpr float kFar = 8.0f;
    auto raise = [&](float m) {                 // to a greater reference
        const float was = a.m;
        if (DT == XGEN_F32) {
            const float d = was == -INFINITY ? 0.0f : was - m, e = exp2_approx(d * kLog2e);
            if (ENTROPY) a.w = e > 0.0f ? (a.w + d * a.s) * e : 0.0f;
            a.s *= e;
            m2 = m;
        } else {
            const float n2 = m * kLog2e, d = was == -INFINITY ? 0.0f : m2 - n2, e = exp2_approx(d);
            if (ENTROPY) a.w = (a.w + d * a.s) * e;
            a.s *= e;
            m2 = n2;
        }
        a.m = m;
    };
    // two elements at a time, as packed fp32
    uint64_t s2 = 0, w2 = 0;
    auto add = [&](float v0, float v1) {
        uint64_t d2;
        float d0, d1;
        if (DT == XGEN_F32) {                   // the difference first: a product of a large logit could overflow
            d2 = add2(pair(v0, v1), pair(-m2, -m2));
            unpair(mul2(d2, pair(kLog2e, kLog2e)), d0, d1);
        } else {
            d2 = fma2(pair(v0, v1), pair(kLog2e, kLog2e), pair(-m2, -m2));
            unpair(d2, d0, d1);
        }
        const uint64_t e2 = pair(exp2_approx(d0), exp2_approx(d1));
        s2 = add2(s2, e2);
        if (ENTROPY) {                          // (e is 0 below -200: so -infinity adds 0, not a NaN)
            unpair(d2, d0, d1);
            w2 = fma2(e2, pair(fmaxf(d0, -200.0f), fmaxf(d1, -200.0f)), w2);
        }
    };
    auto settle = [&] {                         // the packed sums into a
        float x, y;
        unpair(s2, x, y);
        a.s += x + y;
        unpair(w2, x, y);
        a.w += x + y;
        s2 = w2 = 0;
    };
    auto single = [&](int i) {
        const float v = widen(x[i]);
        if (v > own_m) { own_m = v; at_m = i; }
        if (v > a.m + kFar || (a.m == -INFINITY && v > a.m)) { settle(); raise(v); }
        add(v, -INFINITY);
    };
    if (one_head >= 0) single(one_head);
    // two pieces at a time (those behind the end as -infinity), copied three steps ahead; a stretch is `span` such steps
    const int steps = (hi - lo + kAhead * kThreads - 1) / (kAhead * kThreads);
    const int span = max((steps + kStretches - 1) / kStretches, 1);
    int i = lo + tid, stretches = 0;
    float stretch_m = -INFINITY;
    const auto fetch = [&](int stage, int at) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (at + u * kThreads < hi)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(&mem.ring[stage][u][tid])),
                             "l"(body + (int64_t)(at + u * kThreads) * VEC) : "memory");
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int u = 0; u < kStages - 1; ++u) fetch(u, i + u * kAhead * kThreads);
    for (int step = 0, in = 0; step < steps; ++step, i += kAhead * kThreads) {
        Piece<DT> p[kAhead];
        float m[kAhead];
        fetch((step + kStages - 1) % kStages, i + (kStages - 1) * kAhead * kThreads);
        asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (i + u * kThreads < hi) p[u].take(mem.ring[step % kStages][u][tid]);
            else p[u].nothing();
            m[u] = p[u].most();
        }
        const float largest = fmaxf(m[0], m[1]);
        if (largest > own_m) {
            own_m = largest;
            at_m = head + (i + (m[0] == largest ? 0 : kThreads)) * VEC + VEC - 1;
        }
        if (largest > a.m + kFar) {             // (also from -infinity)
            settle();
            raise(largest);
        }
        stretch_m = fmaxf(stretch_m, largest);
        if (++in == span || step == steps - 1) {
            stretch_top[stretches++][tid] = stretch_m;
            stretch_m = -INFINITY;
            in = 0;
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
#pragma unroll
            for (int j = 0; j < VEC; j += 2) add(p[u].at(j), p[u].at(j + 1));
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    if (one_tail >= 0) single(one_tail);
    settle();
    // (of the element that has this key or a greater one)
    const uint64_t own_key = own_m > -INFINITY ? key_of(own_m, (uint32_t)at_m) : kNone;
    if (DT != XGEN_F32 && a.m > -INFINITY) {    // from powers of two, relative to the rounded m2, to powers of e relative to m
        const float off = fmaf(-a.m, kLog2e, m2), e = exp2_approx(off);
        a.w = (a.w + off * a.s) * e * 0.6931471805599453f;
        a.s *= e;
    }
    a = joined(a);
    if (lane == 0) sums[warp] = a;
    lane_top[warp][lane] = own_key;
    __syncthreads();

    // ---- sums and the parts' keys, of the block and of the row
    await(cluster);
    const Sums nothing = {-INFINITY, 0.0f, 0.0f};
    if (warp == 0) {
        const Sums b = joined(lane < kWarps ? sums[lane] : nothing);
        if (lane == 0) {
            if (cluster == 1) all = b;
            else {
                const uint32_t to = far_address(&far_sums[part], 0);
                far_store(to, b.m); far_store(to + 4, b.s); far_store(to + 8, b.w);
            }
        }
    }
    if (warp == 1 && top > 0) {
        uint64_t v = lane_top[0][lane];
#pragma unroll 2
        for (int o = 1; o < kWarps; ++o) v = lane_top[o][lane] > v ? lane_top[o][lane] : v;
        for (int c = 0; c < cluster; ++c) {
            if (cluster == 1) far_lane_top[0][lane] = v;
            else far_store(far_address(&far_lane_top[part][lane], c), v);
        }
    }
    arrive(cluster);
    await(cluster);
    if (top > 0) {
        if (warp == 1) {                        // the top-th largest of the 32 parts' keys
            uint64_t v = far_lane_top[0][lane];
            for (int c = 1; c < cluster; ++c) v = far_lane_top[c][lane] > v ? far_lane_top[c][lane] : v;
            int before = 0;
#pragma unroll 4
            for (int o = 0; o < 32; ++o) {
                const uint64_t u = __shfl_sync(~0u, v, o);
                before += u > v || (u == v && o < lane);
            }
            if (before == top - 1) bound_key = v;
        }
    }
    if (warp == 0 && part == 0 && cluster > 1) {
        const Sums b = joined(lane < cluster ? far_sums[lane] : nothing);
        if (lane == 0) all = b;
    }
    __syncthreads();
    bool overflow = false;
    if (top > 0) {
        const uint64_t bound = bound_key;
        const float bound_value = bound == kNone ? -INFINITY : unordered((uint32_t)(bound >> 32));
        if (own_m >= bound_value && own_m > -INFINITY) {
#pragma unroll 1
            for (int at = 0; at < stretches; ++at)
                if (stretch_top[at][tid] >= bound_value && stretch_top[at][tid] > -INFINITY)
                    queue[atomicAdd(&n_queue, 1)] = (uint16_t)(at * kThreads + tid);
        }
        __syncthreads();
        const auto look = [&](float v, int index) {
            const uint64_t k = key_of(v, (uint32_t)index);
            if (k < bound) return;
            if (cluster == 1) {
                const int at = atomicAdd(&n_found, 1);
                if (at < kRoom) found[at] = k;
            } else {
                const int at = far_add(far_address(&n_found, 0), 1);
                if (at < kRoom) far_store(far_address(&found[at], 0), k);
            }
        };
        // piece `w / n_queue` of queued stretch `w % n_queue`; behind those, the single elements
        const int n_q = n_queue, in_pieces = n_q * span * kAhead;
#pragma unroll 1
        for (int w = tid; w < in_pieces + 2 * VEC; w += kThreads) {
            Piece<DT> p;
            p.nothing();
            int first = 0;
            if (w < in_pieces) {
                const int q = queue[w % n_q], at = lo + q % kThreads + (q / kThreads * span * kAhead + w / n_q) * kThreads;
                if (at < hi) p.load(body + (int64_t)at * VEC);
                first = head + at * VEC;
            } else {
                const int e = w - in_pieces;
                first = e < VEC ? (part == 0 && e < head ? e : -1) : part == cluster - 1 && tail0 + e - VEC < V ? tail0 + e - VEC : -1;
                if (first >= 0) p.one(x[first]);
            }
            unsigned hits = 0;
#pragma unroll
            for (int j = 0; j < VEC; ++j) hits |= p.at(j) >= bound_value && p.at(j) > -INFINITY ? 1u << j : 0u;
            for (; hits; hits &= hits - 1) {
                const int j = __ffs(hits) - 1;
                look(p.any(j), first + j);
            }
        }
        __syncwarp();
        arrive(cluster);
        await(cluster);
        const int n = cluster == 1 ? n_found : far_load(far_address(&n_found, 0));
        overflow = n > kRoom;
        if (overflow) {
            // the block's best element, `top` times over
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
                    for (int u = 0; u < VEC; ++u) see(p.at(u), head + j * VEC + u);
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
                if (tid == 0) {
                    if (cluster == 1) lists[r] = b;
                    else far_store(far_address(&lists[part * kTopMost + r], 0), b);
                }
                if (b != kNone && k == b) k = next_below(b);
                __syncthreads();
            }
        }
        arrive(cluster);                        // (the first block's counter has been read; the lists are there)
        if (part || overflow) await(cluster);
    }

    // ---- the row's answers
    if (part == 0) {
        const Sums r = all;
        const bool bad = isnan(r.s) || r.m == INFINITY;
        const bool empty = !bad && r.m == -INFINITY;
        const float log_s = logf(r.s);
        auto answer = [&](float v) { return bad ? NAN : empty ? -INFINITY : fminf((v - r.m) - log_s, 0.0f); };
        if (tid == 0 && P.logprob) P.logprob[row] = token == -1 ? 0.0f : token < 0 || token >= V ? NAN : answer(token_logit);
        if (ENTROPY && tid == 32) P.entropy[row] = bad ? NAN : empty ? 0.0f : fmaxf(log_s - r.w / r.s, 0.0f);
        auto put = [&](int rank, uint64_t k) {
            P.top_index[row * top + rank] = bad || k == kNone ? -1 : (int)~(uint32_t)k;
            P.top_logprob[row * top + rank] = bad ? NAN : k == kNone ? -INFINITY : answer(unordered((uint32_t)(k >> 32)));
        };
        if (top > 0 && !overflow) {
            const int n = n_found;
            for (int c = tid; c < n; c += kThreads) {
                const uint64_t k = found[c];
                int rank = 0;
#pragma unroll 2
                for (int o = 0; o < n; ++o) rank += found[o] > k;
                if (rank < top) put(rank, k);
            }
            if (tid >= n && tid < top) put(tid, kNone);
        } else if (top > 0) {
            for (int e = tid; e < cluster * kTopMost; e += kThreads) {
                // an element's rank: its place in its own list, and how many of every other list are greater
                const int list = e / kTopMost, at = e % kTopMost;
                if (at >= top) continue;
                const uint64_t k = lists[e];
                int rank = at;
                for (int c = 0; c < cluster; ++c)
                    for (int o = 0; o < top && c != list; ++o) {
                        const uint64_t u = lists[c * kTopMost + o];
                        rank += u > k || (u == kNone && k == kNone && c < list);
                    }
                if (rank < top) put(rank, k);
            }
        }
    }
    if (top > 0 && part == 0 && !overflow) {
        __syncwarp();
        await(cluster);
    }
}

static const void *kernel_for(xgen_dtype t, bool entropy) {
    if (t == XGEN_F32) return entropy ? (const void *)logprobs_kernel<XGEN_F32, true> : (const void *)logprobs_kernel<XGEN_F32, false>;
    return entropy ? (const void *)logprobs_kernel<XGEN_F16_F32ACC, true> : (const void *)logprobs_kernel<XGEN_F16_F32ACC, false>;
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
        bool ok = on.ok;
        for (const bool entropy : {false, true})
            ok = ok && cudaFuncSetAttribute(kernel_for(d->dtype, entropy), cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess &&
                 cudaFuncSetAttribute(kernel_for(d->dtype, entropy), cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Memory)) == cudaSuccess;
        if (!ok) {
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
    const size_t eb = element_bytes(h->d.dtype);
    if (rows && ((size_t)(rows - 1) * stride + h->d.vocab) * eb > (size_t)1 << 62) return XGEN_ERR_SHAPE;       // (2^64 - 2^33 at most)
    if ((logprob != nullptr) != (token != nullptr) || (top != nullptr) != (h->d.top > 0) || (top_logprob != nullptr) != (h->d.top > 0))
        return XGEN_ERR_INVALID_ARG;
    if (!logprob && !entropy && !top) return XGEN_ERR_INVALID_ARG;
    if (rows == 0) return XGEN_OK;
    if (!x) return XGEN_ERR_INVALID_ARG;
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
    // Blocks to a row: as many as give an SM three at most, while a block's part is at least 8 KB.  us with up to 2, 3 and 4 blocks an
    // SM: 37 rows of 128000 fp16 10.8, 10.7, 15.8; 148 of them 18.8, 18.7, 24.7; 100 rows of 32000 fp32 9.7, 8.8, 8.8.
    int cluster = 1;
    while (cluster < 16 && rows * cluster * 2 <= 3 * h->sms && (int64_t)P.vocab * (int64_t)eb / (cluster * 2) >= 8192) cluster *= 2;
    if (rows * cluster > INT32_MAX) return XGEN_ERR_SHAPE;
    OnDevice on(h->device);
    if (!on.ok) return XGEN_ERR_CUDA;
    void *args[] = {&P, &cluster};
    return launch(kernel_for(h->d.dtype, entropy != nullptr), dim3((unsigned)(rows * cluster)),
                  dim3(kThreads), sizeof(Memory), stream, args, cluster);
}

void xgen_logprobs_free(xgen_logprobs_packed *h) { delete h; }

}  // extern "C"
