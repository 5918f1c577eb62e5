// What the kernels of a decoder step share (pp_norm.cu, pp_q4.cu, pp_moe.cu): element types, packed loads and
// stores of eight elements, and the launch with programmatic stream serialization.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <type_traits>

#include "pp.h"

namespace pp {

inline bool is_16bit(int t) { return t == PP_F16 || t == PP_BF16; }
inline bool is_float(int t) { return t == PP_F32 || is_16bit(t); }
inline bool is_8bit(int t) { return t == PP_I8 || t == PP_E4M3; }
inline int type_bytes(int t) { return t == PP_F32 ? 4 : is_16bit(t) ? 2 : 1; }
inline bool aligned_to(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// Whether rows of two matrices share bytes (w: bytes of a row, ld: bytes between rows).  Matrices that lie in one another's gaps
// are told apart where both have one distance or one has one row or none between; others in each other's range count as apart.
inline bool share_bytes(const void* p, int64_t w_p, int64_t ld_p, int64_t rows_p, const void* q, int64_t w_q, int64_t ld_q, int64_t rows_q) {
    if (!p || !q || rows_p < 1 || rows_q < 1) return false;
    if (rows_p == 1 || ld_p == w_p) w_p *= rows_p, ld_p = w_p, rows_p = 1;
    if (rows_q == 1 || ld_q == w_q) w_q *= rows_q, ld_q = w_q, rows_q = 1;
    const int64_t d = (int64_t)(reinterpret_cast<intptr_t>(q) - reinterpret_cast<intptr_t>(p));
    if (d >= (rows_p - 1) * ld_p + w_p || -d >= (rows_q - 1) * ld_q + w_q) return false;
    if (rows_p == 1 && rows_q == 1) return true;
    if (rows_p == 1) return share_bytes(q, w_q, ld_q, rows_q, p, w_p, ld_p, rows_p);
    if (rows_q == 1) {                                       // a row that starts before q's end: the last such one ends behind q's start
        const int64_t last = (d + w_q - 1) / ld_p < rows_p - 1 ? (d + w_q - 1) / ld_p : rows_p - 1;
        return last * ld_p + w_p > d;
    }
    if (ld_p != ld_q) return false;
    const int64_t in = (d % ld_p + ld_p) % ld_p;             // where q's rows start between p's
    return in < w_p || in + w_q > ld_p;
}

// A call's status.  An error of a launch is also kept by the runtime for whoever asks next: that is taken away with it, or the
// next call that looks behind a launch of its own would report this one's.
inline pp_status_t status_of(cudaError_t e) {
    if (e == cudaSuccess) return PP_OK;
    cudaGetLastError();
    return PP_ERR_CUDA;
}

// SMs of the current device, asked for once per device (148 on a whole B200).
inline int sm_count() {
    static int known[64] = {};
    int device = 0, n = 0;
    if (cudaGetDevice(&device) != cudaSuccess) return 148;
    if (device < 64 && known[device]) return known[device];
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device) != cudaSuccess || n < 1) n = 148;
    if (device < 64) known[device] = n;
    return n;
}

// Launch that lets the kernel's prologue overlap the tail of the previous kernel in the stream: the kernel itself
// waits (griddepcontrol.wait) before it reads what that kernel may have written and before it writes anything.
template <typename... P, typename... A>
inline cudaError_t launch_pdl(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t stream, int cluster, A... args) {
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)cluster;
    at[1].val.clusterDim.y = 1;
    at[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cfg.attrs = at;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}

#ifdef __CUDACC__
__device__ __forceinline__ void pdl_release() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(int8_t v) { return (float)v; }
__device__ __forceinline__ float to_float(__nv_fp8_e4m3 v) { return (float)v; }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

template <typename T, int N> struct alignas(sizeof(T) * N > 16 ? 16 : sizeof(T) * N) Pack { T v[N]; };

// N elements in one (or, for eight floats, two) vector accesses; p is aligned to their size (16 bytes at most).
template <typename T, int N> __device__ __forceinline__ void load_vec(float (&f)[N], const T* p) {
    const Pack<T, N> u = *reinterpret_cast<const Pack<T, N>*>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = to_float(u.v[i]);
}
template <typename T, int N> __device__ __forceinline__ void store_vec(T* p, const float (&f)[N]) {
    Pack<T, N> u;
    if constexpr (std::is_same_v<T, float>) {
#pragma unroll
        for (int i = 0; i < N; ++i) u.v[i] = f[i];
    } else {                                                 // two conversions in one instruction
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            if constexpr (std::is_same_v<T, __half>) *reinterpret_cast<__half2*>(u.v + i) = __floats2half2_rn(f[i], f[i + 1]);
            else *reinterpret_cast<__nv_bfloat162*>(u.v + i) = __floats2bfloat162_rn(f[i], f[i + 1]);
        }
    }
    *reinterpret_cast<Pack<T, N>*>(p) = u;
}

// Four 8-bit codes of floats, to nearest even.
__device__ __forceinline__ uint32_t four_codes(const float* v, bool e4m3) {
    if (e4m3) {
        const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(v[0], v[1]), __NV_SATFINITE, __NV_E4M3);
        const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(v[2], v[3]), __NV_SATFINITE, __NV_E4M3);
        return lo | (hi << 16);
    }
    uint32_t u = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) u |= (uint32_t)(__float2int_rn(fminf(fmaxf(v[i], -127.0f), 127.0f)) & 255) << (8 * i);
    return u;
}
#endif

}  // namespace pp
