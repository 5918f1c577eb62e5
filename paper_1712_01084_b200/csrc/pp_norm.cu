// Root-mean-square normalisation with the residual's addition and a result in 8 bits with scales.
//
//   h = x + r          (written back as the next residual, rounded once to the type of x)
//   n = h * rsqrt(mean(h^2) + eps) * w
//   s = max|n| / Q     over the row, or over each 128 columns of it;  Q = 127 (integers) or 448 (e4m3)
//   q = round(n / s)   to nearest even
//
// One pass: a row's h stays in registers as floats.  max|n| = rsqrt(...) * max|h w|, so the sum of squares and the largest
// |h w| need nothing from each other and one barrier serves both.
//
// Few rows: a CTA per row (rmsnorm_q8_kernel), bound by the latency of one trip to memory.  Many rows: CTAs that stay
// (rmsnorm_q8_rows_kernel), each with a ring of rows on their way into shared memory by 16-byte asynchronous copies while
// it works on the one before; a CTA per row stops the flow of bytes at every barrier.
//
// 8192 x 8192 bf16 with a residual: 76 us in a graph, 6.1 TB/s (80 us called one after another).  One row of 4096: 2.0 us.
// 33 x 9216 to integers: 3.7 us.  2047 x 4095, whose rows start on any two bytes: 18.7 us, bound by 2-byte accesses.
#include <algorithm>

#include "pp_decode.cuh"
#include "pp_internal.h"

namespace pp {
namespace {

struct NormArgs {
    const void *x, *r, *w;
    void *codes, *hidden, *normed;
    float* scales;
    int64_t ldx, ldr, ldh;
    int cols, n_groups;
    float eps, per_col;                      // 1 / cols
    int w_f32, rows, stage_bytes;            // the last two: of the kernel for many rows
};

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// The larger of two, a NaN before all: fmaxf would drop it, and an infinity times a weight of 0 is one.
__device__ __forceinline__ float max_nan(float a, float b) {
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
// Largest of a warp's, or of each half warp's, values >= 0 (which order as whole numbers do; a NaN is the largest).
template <int W> __device__ __forceinline__ float lanes_max(float v) {
    if (W == 32) return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(v)));
#pragma unroll
    for (int o = W / 2; o; o >>= 1) v = max_nan(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// Column of element i (0..7) of this thread's chunk c.  A warp owns 256 consecutive columns of a chunk.  VEC: eight
// neighbours per thread, half a warp to a group of 128.  Otherwise a warp's accesses are 32 neighbours, elements
// 0..3 of all its lanes are the first group and 4..7 the second.
template <bool VEC> __device__ __forceinline__ int column(int c, int i) {
    const int base = (c * blockDim.x + (threadIdx.x & ~31)) * 8, lane = threadIdx.x & 31;
    return base + (VEC ? lane * 8 + i : i * 32 + lane);
}

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

// The weights of this thread's chunk c as floats, 0 past the row's end.
template <typename T, bool VEC> __device__ __forceinline__ void load_weights(const NormArgs& a, int c, float (&w)[8]) {
    const int j0 = column<VEC>(c, 0);
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = 0.0f;
    if (VEC) {
        if (j0 < a.cols) {
            if (a.w_f32) load_vec(w, static_cast<const float*>(a.w) + j0);
            else load_vec(w, static_cast<const T*>(a.w) + j0);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int j = j0 + 32 * i;
            if (j < a.cols) w[i] = a.w_f32 ? static_cast<const float*>(a.w)[j] : to_float(static_cast<const T*>(a.w)[j]);
        }
    }
}

// From a row's h in registers to everything that is written of it.  weights(c, w): those of chunk c; part: [2][32] floats that
// the row before did not use.
template <typename T, int CH, bool VEC, bool GROUPED, bool E4M3, typename Weights>
__device__ __forceinline__ void finish_row(const NormArgs& a, int64_t row, float (&h)[CH][8], Weights weights, float* part) {
    constexpr float kTop = E4M3 ? 448.0f : 127.0f;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = blockDim.x >> 5;
    T* hidden = a.hidden ? static_cast<T*>(a.hidden) + row * a.ldh : nullptr;
    float top[CH][2], sum = 0.0f, most = 0.0f;               // top: the largest |h w| of the chunk's first and second group
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int j0 = column<VEC>(c, 0);
        if (hidden) {
            if (VEC) {
                if (j0 < a.cols) store_vec(hidden + j0, h[c]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (j0 + 32 * i < a.cols) hidden[j0 + 32 * i] = from_float<T>(h[c][i]);
            }
        }
        top[c][0] = top[c][1] = 0.0f;
        float w[8];
        weights(c, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) {                        // h and w are 0 past the row's end
            sum = fmaf(h[c][i], h[c][i], sum);
            h[c][i] *= w[i];
            top[c][!VEC && i >= 4] = max_nan(top[c][!VEC && i >= 4], fabsf(h[c][i]));
        }
        if (GROUPED) {
            if (VEC) {
                top[c][0] = lanes_max<16>(top[c][0]);
            } else {
                top[c][0] = lanes_max<32>(top[c][0]);
                top[c][1] = lanes_max<32>(top[c][1]);
            }
        } else {
            most = max_nan(most, max_nan(top[c][0], top[c][1]));
        }
    }
    sum = warp_sum(sum);
    if (!GROUPED) most = lanes_max<32>(most);
    if (lane == 0) {
        part[warp] = sum;
        part[32 + warp] = most;
    }
    __syncthreads();
    sum = warp_sum(lane < n_warps ? part[lane] : 0.0f);
    if (!GROUPED) most = lanes_max<32>(lane < n_warps ? part[32 + lane] : 0.0f);
    // a sum that is not finite (an element that is not, or squares beyond fp32) makes every scale of the row NaN: the root's 0
    // would make them 0
    const float rms = sum < INFINITY ? rsqrtf(fmaf(sum, a.per_col, a.eps)) : __int_as_float(0x7fffffff);

    uint8_t* codes = static_cast<uint8_t*>(a.codes) + row * a.cols;
    if (!GROUPED && threadIdx.x == 0) a.scales[row] = rms * most * (1.0f / kTop);
    if (a.normed) {
        T* normed = static_cast<T*>(a.normed) + row * a.cols;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int j0 = column<VEC>(c, 0);
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = h[c][i] * rms;
            if (VEC) {
                if (j0 < a.cols) store_vec(normed + j0, v);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (j0 + 32 * i < a.cols) normed[j0 + 32 * i] = from_float<T>(v[i]);
            }
        }
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int j0 = column<VEC>(c, 0);
        float v[8];
#pragma unroll
        for (int g = 0; g < (!VEC && GROUPED ? 2 : 1); ++g) {
            // n / s = (h w) * Q / max|h w|: one multiplication per element; far from 1 both are brought nearer by 2^64 first, so
            // that the quotient neither overflows nor leaves the range of the fast division
            float of = GROUPED ? top[c][g] : most;
            const float largest = rms * of;
            if (GROUPED && (VEC ? (lane & 15) == 0 : lane == 0)) {
                const int group = VEC ? j0 / 128 : (j0 / 128) + g;
                if (group < a.n_groups) a.scales[row * a.n_groups + group] = largest * (1.0f / kTop);
            }
            if (of < 0x1p-60f || of > 0x1p60f) {
                const float near = of < 1.0f ? 0x1p64f : 0x1p-64f;
                of *= near;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (VEC || !GROUPED || i / 4 == g) h[c][i] *= near;
            }
            const float m = largest > 0.0f ? __fdividef(kTop, of) : 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (VEC || !GROUPED || i / 4 == g) v[i] = h[c][i] * m;
        }
        const uint32_t q0 = four_codes(v, E4M3), q1 = four_codes(v + 4, E4M3);
        if (VEC) {
            if (j0 < a.cols) *reinterpret_cast<uint2*>(codes + j0) = make_uint2(q0, q1);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (j0 + 32 * i < a.cols) codes[j0 + 32 * i] = (uint8_t)((i < 4 ? q0 : q1) >> (8 * (i & 3)));
        }
    }
}

template <typename T, int CH, bool VEC, bool GROUPED, bool E4M3>
__global__ void __launch_bounds__(1024) rmsnorm_q8_kernel(const NormArgs a) {
    __shared__ float part[64];
    pdl_release();
    pdl_wait();
    const int64_t row = blockIdx.x;
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    const T* r = a.r ? static_cast<const T*>(a.r) + row * a.ldr : nullptr;
    float h[CH][8];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int j0 = column<VEC>(c, 0);
#pragma unroll
        for (int i = 0; i < 8; ++i) h[c][i] = 0.0f;
        if (VEC) {
            if (j0 < a.cols) load_vec(h[c], x + j0);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (j0 + 32 * i < a.cols) h[c][i] = to_float(x[j0 + 32 * i]);
        }
    }
    if (r) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int j0 = column<VEC>(c, 0);
            if (VEC) {
                if (j0 < a.cols) {
                    float v[8];
                    load_vec(v, r + j0);
#pragma unroll
                    for (int i = 0; i < 8; ++i) h[c][i] += v[i];
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (j0 + 32 * i < a.cols) h[c][i] += to_float(r[j0 + 32 * i]);
            }
        }
    }
    // a thread has read every x and r it will ever read before it writes: hidden may be either of them
    finish_row<T, CH, VEC, GROUPED, E4M3>(a, row, h, [&](int c, float (&w)[8]) { load_weights<T, VEC>(a, c, w); }, part);
}

// Rows in the ring of a CTA, and the columns of a thread: 32, so that what a row costs each thread beside its elements (two
// reductions, one barrier) is spread over many (8192 x 8192 bf16: 8 columns a thread 99 us, 16 86 us, 32 80 us; a CTA per row
// 92 us.  With rows counted without a sign 32 take 76, with 64-bit numbers 83).
constexpr int kStages = 3, kRowsChunks = 4, kRowsThreads = 320;

// Rows that start on 16 bytes (VEC): a thread reads only what it has copied itself.
template <typename T, bool GROUPED, bool E4M3>
__global__ void __launch_bounds__(kRowsThreads, 2) rmsnorm_q8_rows_kernel(const NormArgs a) {
    constexpr int CH = kRowsChunks;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float part[2][64];
    const int half = a.stage_bytes / 2;                      // x, then r
    pdl_release();
    pdl_wait();
    float w[CH][8];
#pragma unroll
    for (int c = 0; c < CH; ++c) load_weights<T, true>(a, c, w[c]);
    const T *x = static_cast<const T*>(a.x), *r = static_cast<const T*>(a.r);
    const auto fetch = [&](uint32_t row, int stage) {
        if (row < (uint32_t)a.rows) {
            const uint32_t dst = (uint32_t)__cvta_generic_to_shared(smem + stage * a.stage_bytes);
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int j0 = column<true>(c, 0);
                if (j0 >= a.cols) break;
#pragma unroll
                for (int i = 0; i < 8; i += 16 / (int)sizeof(T)) {
                    const uint32_t at = dst + (j0 + i) * (int)sizeof(T);
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at), "l"(x + row * a.ldx + j0 + i));
                    if (r) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at + half), "l"(r + row * a.ldr + j0 + i));
                }
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    const uint32_t step = gridDim.x, rows = (uint32_t)a.rows;        // rows asked for ahead may pass 2^31
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) fetch(blockIdx.x + s * step, s);
    int stage = 0, parity = 0;
    for (uint32_t row = blockIdx.x; row < rows; row += step) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
        const unsigned char* at = smem + stage * a.stage_bytes;
        float h[CH][8];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int j0 = column<true>(c, 0);
#pragma unroll
            for (int i = 0; i < 8; ++i) h[c][i] = 0.0f;
            if (j0 < a.cols) {
                load_vec(h[c], reinterpret_cast<const T*>(at) + j0);
                if (r) {
                    float v[8];
                    load_vec(v, reinterpret_cast<const T*>(at + half) + j0);
#pragma unroll
                    for (int i = 0; i < 8; ++i) h[c][i] += v[i];
                }
            }
        }
        int ahead = stage + kStages - 1;                     // the stage that the row before has left
        if (ahead >= kStages) ahead -= kStages;
        fetch(row + (kStages - 1) * step, ahead);
        finish_row<T, CH, true, GROUPED, E4M3>(a, row, h, [&](int c, float (&v)[8]) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = w[c][i];
        }, part[parity]);
        parity ^= 1;
        if (++stage == kStages) stage = 0;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
}

template <typename T, int CH, bool VEC>
cudaError_t launch(const NormArgs& a, int threads, bool grouped, bool e4m3, cudaStream_t stream) {
    auto k = grouped ? (e4m3 ? rmsnorm_q8_kernel<T, CH, VEC, true, true> : rmsnorm_q8_kernel<T, CH, VEC, true, false>)
                     : (e4m3 ? rmsnorm_q8_kernel<T, CH, VEC, false, true> : rmsnorm_q8_kernel<T, CH, VEC, false, false>);
    return launch_pdl(k, dim3(a.rows), dim3(threads), 0, stream, 1, a);
}

template <typename T> cudaError_t launch_rows(const NormArgs& a, int grid, int threads, bool grouped, bool e4m3, cudaStream_t stream) {
    static PerDeviceOnce opt_in[2][2];
    auto k = grouped ? (e4m3 ? rmsnorm_q8_rows_kernel<T, true, true> : rmsnorm_q8_rows_kernel<T, true, false>)
                     : (e4m3 ? rmsnorm_q8_rows_kernel<T, false, true> : rmsnorm_q8_rows_kernel<T, false, false>);
    PerDeviceOnce& once = opt_in[grouped][e4m3];
    int device = 0;
    if (cudaError_t e = cudaGetDevice(&device)) return e;
    if (!once.is_done(device)) {
        if (cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, 226 * 1024)) return e;
        once.mark(device);
    }
    return launch_pdl(k, dim3(grid), dim3(threads), (size_t)kStages * a.stage_bytes, stream, 1, a);
}

template <typename T>
cudaError_t launch_type(NormArgs& a, bool vec, bool grouped, bool e4m3, cudaStream_t stream) {
    // Many rows: as many staying CTAs as an SM's shared memory and registers (96 a thread) take, if each then has four rows
    // (1024 x 4096, under two rows each: 8.0 us against 6.8 of a CTA per row; 1200 x 8192, four rows: 15.1 against 16.8).
    const int staying = ((a.cols + 8 * kRowsChunks - 1) / (8 * kRowsChunks) + 31) / 32 * 32;
    a.stage_bytes = 2 * (int)(((size_t)a.cols * sizeof(T) + 15) / 16 * 16);
    const int each = std::min({680 / staying, (227 * 1024) / (kStages * a.stage_bytes + 2048), 16});
    if (vec && staying <= kRowsThreads && each >= 1) {
        const int grid = sm_count() * each;
        if (a.rows >= 4 * grid) return launch_rows<T>(a, grid, staying, grouped, e4m3, stream);
    }
    // as few columns per thread as 1024 threads allow: the row's latency is one trip to memory either way
    int ch = 1;
    while (ch < 4 && a.cols > 1024 * 8 * ch) ch *= 2;
    const int threads = ((a.cols + 8 * ch - 1) / (8 * ch) + 31) / 32 * 32;
    switch (ch * 2 + vec) {
        case 2: return launch<T, 1, false>(a, threads, grouped, e4m3, stream);
        case 3: return launch<T, 1, true>(a, threads, grouped, e4m3, stream);
        case 4: return launch<T, 2, false>(a, threads, grouped, e4m3, stream);
        case 5: return launch<T, 2, true>(a, threads, grouped, e4m3, stream);
        case 8: return launch<T, 4, false>(a, threads, grouped, e4m3, stream);
        default: return launch<T, 4, true>(a, threads, grouped, e4m3, stream);
    }
}

}  // namespace
}  // namespace pp

extern "C" pp_status_t pp_rmsnorm_q8(const void* x, int64_t ldx, const void* residual, int64_t ldr, const void* weight,
                                     pp_dtype_t dtype, pp_dtype_t weight_type, int rows, int cols, float eps,
                                     pp_dtype_t code_type, int group, void* codes, float* scales, void* hidden_out,
                                     int64_t ldh, void* normed_out, void* cuda_stream) {
    using namespace pp;
    if (rows < 0 || cols < 1 || !(eps >= 0.0f) || (rows > 0 && (!x || !weight || !codes || !scales))) return PP_ERR_INVALID_ARG;
    if (!is_float(dtype) || (weight_type != dtype && weight_type != PP_F32) || !is_8bit(code_type)) return PP_ERR_UNSUPPORTED;
    if (group != 0 && group != 128) return PP_ERR_UNSUPPORTED;
    if (cols > 32768) return PP_ERR_UNSUPPORTED;
    if (rows > 1 && (ldx < cols || (residual && ldr < cols) || (hidden_out && ldh < cols))) return PP_ERR_INVALID_ARG;
    const size_t tb = (size_t)type_bytes(dtype);
    if (!aligned_to(x, tb) || !aligned_to(residual, tb) || !aligned_to(hidden_out, tb) || !aligned_to(normed_out, tb) ||
        !aligned_to(weight, (size_t)type_bytes(weight_type)) || !aligned_to(scales, 4)) return PP_ERR_INVALID_ARG;
    if (rows == 0) return PP_OK;
    const int64_t width = (int64_t)cols * (int64_t)tb;
    const auto crosses_hidden = [&](const void* p, int64_t ld) {          // over it but not in its place
        return share_bytes(p, width, ld * (int64_t)tb, rows, hidden_out, width, ldh * (int64_t)tb, rows) && !(p == hidden_out && (rows == 1 || ld == ldh));
    };
    if (crosses_hidden(x, ldx) || crosses_hidden(residual, ldr)) return PP_ERR_INVALID_ARG;
    NormArgs a{x, residual, weight, codes, hidden_out, normed_out, scales, ldx, ldr, ldh,
               cols, group ? (cols + 127) / 128 : 1, eps, 1.0f / (float)cols, weight_type == PP_F32, rows, 0};
    // eight elements to an access where every row of every array starts on one
    const auto rows16 = [&](const void* p, int64_t ld) { return !p || (aligned_to(p, 16) && (rows == 1 || ld * (int64_t)tb % 16 == 0)); };
    const bool vec = cols % 8 == 0 && rows16(x, ldx) && rows16(residual, ldr) && rows16(hidden_out, ldh) && rows16(normed_out, cols) &&
                     aligned_to(weight, 16) && aligned_to(codes, 8);
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    const cudaError_t e = dtype == PP_F32 ? launch_type<float>(a, vec, group != 0, code_type == PP_E4M3, s)
                        : dtype == PP_F16 ? launch_type<__half>(a, vec, group != 0, code_type == PP_E4M3, s)
                                          : launch_type<__nv_bfloat16>(a, vec, group != 0, code_type == PP_E4M3, s);
    return status_of(e);
}
