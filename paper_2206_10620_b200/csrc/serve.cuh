// What the operators between the products share: launches, element access, warp matrix products.
#pragma once
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "patconv_internal.h"

namespace serve {

// The handle's device is current while one of these lives.
struct OnDevice {
    int prev = -1;
    bool ok = true;
    explicit OnDevice(int device) {
        int now = -1;
        if (cudaGetDevice(&now) != cudaSuccess) { cudaGetLastError(); ok = false; return; }
        if (now == device) return;
        if (cudaSetDevice(device) != cudaSuccess) { cudaGetLastError(); ok = false; return; }
        prev = now;
    }
    ~OnDevice() { if (prev >= 0) cudaSetDevice(prev); }
    OnDevice(const OnDevice &) = delete;
};

// One launch on the caller's stream.  The kernel may start while its predecessor ends: it calls wait_before() ahead of its
// first access to memory that the predecessor could write or still read, and reads none of it by read-only loads (__ldg): those are for
// what nobody writes while the kernel lives, and it lives while its predecessor writes.  cluster: blocks along x that form one, or 1.
inline xgen_status launch(const void *kern, dim3 grid, dim3 block, size_t shared, void *stream, void **args, int cluster = 1) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid; cfg.blockDim = block; cfg.dynamicSmemBytes = shared; cfg.stream = (cudaStream_t)stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = cluster > 1 ? 2 : 1;
    if (cudaLaunchKernelExC(&cfg, kern, args) != cudaSuccess) {
        cudaGetLastError();
        return XGEN_ERR_CUDA;
    }
    patconv::count_launch();
    return XGEN_OK;
}

// Whether [a, a + an) and [b, b + bn) share a byte (of addresses that do not end: a span may be longer than what is left of them).
inline bool overlap(const void *a, size_t an, const void *b, size_t bn) {
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return a && b && an && bn && (x < y ? y - x < an : x - y < bn);
}

// The stream's work done, whether the kernels left a mark at `mark` (marks[0]: an argument that does not fit; marks[1], where there are two: a
// wait that ran out); marks are taken away again.
inline xgen_status take_status(int device, int *marks, int count, void *stream) {
    OnDevice on(device);
    int seen[2] = {0, 0};
    const cudaStream_t st = (cudaStream_t)stream;
    if (!on.ok || cudaStreamSynchronize(st) != cudaSuccess || cudaMemcpyAsync(seen, marks, 4 * count, cudaMemcpyDeviceToHost, st) != cudaSuccess ||
        cudaStreamSynchronize(st) != cudaSuccess ||
        ((seen[0] || seen[1]) && (cudaMemsetAsync(marks, 0, 4 * count, st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess))) {
        cudaGetLastError();
        return XGEN_ERR_CUDA;
    }
    return seen[1] ? XGEN_ERR_TIMEOUT : seen[0] ? XGEN_ERR_INVALID_ARG : XGEN_OK;
}
inline size_t element_bytes(xgen_dtype t) { return t == XGEN_F32 ? 4 : 2; }

#ifdef __CUDACC__

__device__ __forceinline__ void wait_before() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// From here on (every block has to get there, or end) the next launch on the stream may take what room there is.
__device__ __forceinline__ void let_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

template <int DT> struct Elem;
template <> struct Elem<XGEN_F32> { using T = float; };
template <> struct Elem<XGEN_F16_F32ACC> { using T = __half; };
__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T narrow(float v);
template <> __device__ __forceinline__ float narrow<float>(float v) { return v; }
template <> __device__ __forceinline__ __half narrow<__half>(float v) { return __float2half_rn(v); }

// One matrix instruction of a warp: D[16][8] += A[16][16] B[16][8], fp16 in, fp32 sums.  Lane 4g + t holds of A the rows g
// (a[0], a[2]) and g + 8 (a[1], a[3]), columns 2t, 2t+1 (a[0], a[1]) and 2t+8, 2t+9; of B column g, rows 2t, 2t+1
// and 2t+8, 2t+9; of D rows g (d[0], d[1]) and g + 8, columns 2t, 2t+1.
__device__ __forceinline__ void mma16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// The same with fp32 operands cut to tf32 by the unit: A[16][8] (rows g, g + 8; columns t (a[0], a[1]) and t + 4), B[8][8]
// (rows t, t + 4).
__device__ __forceinline__ void mma_tf32(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// 2^e for an exponent within -126 .. 127.
__device__ __forceinline__ float pow2(int e) { return __int_as_float((e + 127) << 23); }
// The exponent of a finite magnitude above 0 (that of a subnormal one reads as -127).
__device__ __forceinline__ int exponent(float v) { return (int)((__float_as_uint(v) >> 23) & 255u) - 127; }
__device__ __forceinline__ float exp2_approx(float v) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// Two fp32 numbers in one register pair, and what one instruction does to both.
__device__ __forceinline__ uint64_t pair(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpair(uint64_t v, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

#endif  // __CUDACC__
}  // namespace serve
