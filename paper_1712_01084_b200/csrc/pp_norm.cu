// Root-mean-square normalisation with the residual's addition and a result in 8 bits with scales.
//
//   h = x + r          (written back as the next residual, rounded once to the type of x)
//   n = h * rsqrt(mean(h^2) + eps) * w
//   s = max|n| / Q     over the row, or over each 128 columns of it;  Q = 127 (integers) or 448 (e4m3)
//   q = round(n / s)   to nearest even
//
// One CTA per row and one pass: the row's h stays in registers as floats.  max|n| = rsqrt(...) * max|h w|, so the
// sum of squares and the largest |h w| need nothing from each other and one barrier serves both.
#include "pp_decode.cuh"

namespace pp {
namespace {

struct NormArgs {
    const void *x, *r, *w;
    void *codes, *hidden, *normed;
    float* scales;
    int64_t ldx, ldr, ldh;
    int cols, n_groups;
    float eps;
    int w_f32;
};

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
template <int W> __device__ __forceinline__ float lanes_max(float v) {
#pragma unroll
    for (int o = W / 2; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
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

template <typename T, int CH, bool VEC, bool GROUPED, bool E4M3>
__global__ void __launch_bounds__(1024) rmsnorm_q8_kernel(const NormArgs a) {
    constexpr float kTop = E4M3 ? 448.0f : 127.0f;
    __shared__ float part[2][32];
    pdl_release();
    pdl_wait();
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = blockDim.x >> 5;
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    const T* r = a.r ? static_cast<const T*>(a.r) + row * a.ldr : nullptr;

    float h[CH][8], top[CH][2], sum = 0.0f, most = 0.0f;     // top: the largest |h w| of the chunk's first and second group
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int j0 = column<VEC>(c, 0);
        if (VEC) {
            if (j0 < a.cols) {
                load_vec(h[c], x + j0);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) h[c][i] = 0.0f;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) h[c][i] = j0 + 32 * i < a.cols ? to_float(x[j0 + 32 * i]) : 0.0f;
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
    T* hidden = a.hidden ? static_cast<T*>(a.hidden) + row * a.ldh : nullptr;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int j0 = column<VEC>(c, 0);
        float w[8];
        if (VEC) {
            if (j0 < a.cols) {
                if (a.w_f32) load_vec(w, static_cast<const float*>(a.w) + j0);
                else load_vec(w, static_cast<const T*>(a.w) + j0);
                if (hidden) store_vec(hidden + j0, h[c]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int j = j0 + 32 * i;
                w[i] = j >= a.cols ? 0.0f : a.w_f32 ? static_cast<const float*>(a.w)[j] : to_float(static_cast<const T*>(a.w)[j]);
                if (hidden && j < a.cols) hidden[j] = from_float<T>(h[c][i]);
            }
        }
        top[c][0] = top[c][1] = 0.0f;
        if (j0 < a.cols) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                sum = fmaf(h[c][i], h[c][i], sum);
                h[c][i] *= w[i];
                top[c][!VEC && i >= 4] = fmaxf(top[c][!VEC && i >= 4], fabsf(h[c][i]));
            }
        }
        if (GROUPED) {
            if (VEC) {
                top[c][0] = lanes_max<16>(top[c][0]);
            } else {
                top[c][0] = lanes_max<32>(top[c][0]);
                top[c][1] = lanes_max<32>(top[c][1]);
            }
        } else {
            most = fmaxf(most, fmaxf(top[c][0], top[c][1]));
        }
    }
    sum = warp_sum(sum);
    if (!GROUPED) most = lanes_max<32>(most);
    if (lane == 0) {
        part[0][warp] = sum;
        part[1][warp] = most;
    }
    __syncthreads();
    sum = warp_sum(lane < n_warps ? part[0][lane] : 0.0f);
    if (!GROUPED) most = lanes_max<32>(lane < n_warps ? part[1][lane] : 0.0f);
    const float rms = rsqrtf(sum / (float)a.cols + a.eps);

    uint8_t* codes = static_cast<uint8_t*>(a.codes) + row * a.cols;
    T* normed = a.normed ? static_cast<T*>(a.normed) + row * a.cols : nullptr;
    if (!GROUPED && threadIdx.x == 0) a.scales[row] = rms * most / kTop;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int j0 = column<VEC>(c, 0);
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = h[c][i] * rms;
        if (normed) {
            if (VEC) {
                if (j0 < a.cols) store_vec(normed + j0, v);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (j0 + 32 * i < a.cols) normed[j0 + 32 * i] = from_float<T>(v[i]);
            }
        }
#pragma unroll
        for (int g = 0; g < (!VEC && GROUPED ? 2 : 1); ++g) {
            const float s = rms * (GROUPED ? top[c][g] : most) / kTop;
            if (GROUPED && (VEC ? (lane & 15) == 0 : lane == 0)) {
                const int group = VEC ? j0 / 128 : (j0 / 128) + g;
                if (group < a.n_groups) a.scales[row * a.n_groups + group] = s;
            }
            // n / s by one reciprocal; a scale so small that its reciprocal overflows divides, and 0 codes as 0
            const float inv = s > 0.0f ? 1.0f / s : s == 0.0f ? 0.0f : s;
            const bool tiny = isinf(inv);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (VEC || !GROUPED || i / 4 == g) v[i] = tiny ? v[i] / s : v[i] * inv;
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

template <typename T, int CH, bool VEC>
cudaError_t launch(const NormArgs& a, int rows, int threads, bool grouped, bool e4m3, cudaStream_t stream) {
    auto k = grouped ? (e4m3 ? rmsnorm_q8_kernel<T, CH, VEC, true, true> : rmsnorm_q8_kernel<T, CH, VEC, true, false>)
                     : (e4m3 ? rmsnorm_q8_kernel<T, CH, VEC, false, true> : rmsnorm_q8_kernel<T, CH, VEC, false, false>);
    return launch_pdl(k, dim3(rows), dim3(threads), 0, stream, 1, a);
}

template <typename T>
cudaError_t launch_type(const NormArgs& a, int rows, bool vec, bool grouped, bool e4m3, cudaStream_t stream) {
    // as few columns per thread as 1024 threads allow: the row's latency is one trip to memory either way
    int ch = 1;
    while (ch < 4 && a.cols > 1024 * 8 * ch) ch *= 2;
    const int threads = ((a.cols + 8 * ch - 1) / (8 * ch) + 31) / 32 * 32;
    switch (ch * 2 + vec) {
        case 2: return launch<T, 1, false>(a, rows, threads, grouped, e4m3, stream);
        case 3: return launch<T, 1, true>(a, rows, threads, grouped, e4m3, stream);
        case 4: return launch<T, 2, false>(a, rows, threads, grouped, e4m3, stream);
        case 5: return launch<T, 2, true>(a, rows, threads, grouped, e4m3, stream);
        case 8: return launch<T, 4, false>(a, rows, threads, grouped, e4m3, stream);
        default: return launch<T, 4, true>(a, rows, threads, grouped, e4m3, stream);
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
    NormArgs a{x, residual, weight, codes, hidden_out, normed_out, scales, ldx, ldr, ldh,
               cols, group ? (cols + 127) / 128 : 1, eps, weight_type == PP_F32};
    // eight elements to an access where every row of every array starts on one
    const auto rows16 = [&](const void* p, int64_t ld) { return !p || (aligned_to(p, 16) && (rows == 1 || ld * (int64_t)tb % 16 == 0)); };
    const bool vec = cols % 8 == 0 && rows16(x, ldx) && rows16(residual, ldr) && rows16(hidden_out, ldh) && rows16(normed_out, cols) &&
                     aligned_to(weight, 16) && aligned_to(codes, 8);
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    const cudaError_t e = dtype == PP_F32 ? launch_type<float>(a, rows, vec, group != 0, code_type == PP_E4M3, s)
                        : dtype == PP_F16 ? launch_type<__half>(a, rows, vec, group != 0, code_type == PP_E4M3, s)
                                          : launch_type<__nv_bfloat16>(a, rows, vec, group != 0, code_type == PP_E4M3, s);
    return e == cudaSuccess ? PP_OK : PP_ERR_CUDA;
}
