// y = act(W x + b) with 4-bit weights and group scales, for a few input vectors: layout (pp_q4.cuh), the kernel that
// rewrites plain codes into units, the product, and the C entry points.
//
// The product reads every weight once, so it is bound by HBM for large matrices and by the latency of one launch for
// small ones.  A cluster of S CTAs owns a run of 16-row strips; its CTAs own S equal parts of the columns, so each
// stages only its part of x.  A CTA's units, strip after strip, are dealt to its 16 warps in equal contiguous runs;
// every warp keeps a ring of units in flight in shared memory with 16-byte asynchronous copies, requested before the
// wait for the previous kernel (weights are never written by a kernel).  Partial sums meet in shared memory, those of
// the other CTAs arrive there through the cluster's distributed shared memory; all are added in one fixed order.
#include "pp_q4.cuh"

#include <algorithm>
#include <new>

struct pp_q4 {
    int M, N, group, sets, strips, blocks;
    bool asym, bf16_scales;
    unsigned char* units;
    float* bias;
    int max_clusters[9];      // clusters of this size that the device holds at once
};

namespace pp {
namespace {

constexpr int kWarps = 16, kThreads = kWarps * 32, kDepth = 4, kMaxStrips = 16, kMaxCols = 32;

struct Q4Args {
    const unsigned char* units;
    const float* bias;
    XIn in;
    void* y;
    int64_t ldy;
    int y_type, act, tokens, nc;          // nc: columns of the staged input = tokens * columns_per_token
    int M, strips, blocks, unit_bytes, bf16_scales;
    int ring_off, cs_off, park_off, red_off;      // shared memory; the staged input is at 0
};

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void st_cluster(uint32_t local, uint32_t rank, float v) {
    uint32_t remote;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(local), "r"(rank));
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(remote), "f"(v) : "memory");
}

__device__ __forceinline__ void store_y(void* y, int64_t i, int type, float v) {
    if (type == PP_F32) static_cast<float*>(y)[i] = v;
    else if (type == PP_F16) static_cast<__half*>(y)[i] = __float2half_rn(v);
    else static_cast<__nv_bfloat16*>(y)[i] = __float2bfloat16_rn(v);
}

template <int NT, int SETS, bool ASYM>
__global__ void __launch_bounds__(kThreads, NT == 1 ? 2 : 1) q4_kernel(const Q4Args a) {
    extern __shared__ __align__(128) unsigned char smem[];
    const int S = (int)cluster_size(), rank = (int)cluster_rank();
    const int n_clusters = gridDim.x / S, cl = blockIdx.x / S;
    const int s0 = (int)((int64_t)a.strips * cl / n_clusters), n_s = (int)((int64_t)a.strips * (cl + 1) / n_clusters) - s0;
    const int k0 = a.blocks * rank / S, n_k = a.blocks * (rank + 1) / S - k0;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int U = n_s * n_k, u0 = U * warp / kWarps, u1 = U * (warp + 1) / kWarps;
    if (S > 1) asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
    pdl_release();

    // the first units of this warp: nothing in them depends on an earlier kernel
    const int extra16 = SETS * (ASYM ? 3 : 2);
    const uint32_t ring = smem_addr(smem + a.ring_off) + (uint32_t)(warp * kDepth * a.unit_bytes);
    int fs = n_k ? u0 / n_k : 0, fk = n_k ? u0 - fs * n_k : 0, fetched = u0;
    const unsigned char* src = a.units + ((int64_t)(s0 + fs) * a.blocks + k0 + fk) * a.unit_bytes;
    auto fetch = [&](uint32_t slot) {
        if (fetched < u1) {
            q4_fetch(slot, src, lane, extra16);
            ++fetched;
            src += a.unit_bytes;
            if (++fk == n_k) {
                fk = 0;
                src += (int64_t)(a.blocks - n_k) * a.unit_bytes;
            }
        }
        cp_commit();
    };
#pragma unroll
    for (int d = 0; d < kDepth; ++d) fetch(ring + d * a.unit_bytes);

    pdl_wait();
    // stage this CTA's columns of x: [32 columns][column of the tile][32 halves]
    __half* xs = reinterpret_cast<__half*>(smem);
    float* cs = reinterpret_cast<float*>(smem + a.cs_off);
    const int step = a.nc * 32, cpt = columns_per_token(a.in.type), items = a.tokens * n_k;
    for (int base = warp; base < items; base += 4 * kWarps) {
        float v[4][4];
        int tok[4], kb[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int item = base + q * kWarps;
            tok[q] = item / n_k;
            kb[q] = item - tok[q] * n_k;
            if (item < items) load_four(v[q], a.in, (int64_t)tok[q] * a.in.ld, (k0 + kb[q]) * kQ4UnitCols + lane * 4);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (base + q * kWarps < items) {
                const float down = stage_block(v[q], a.in, tok[q], k0 + kb[q], xs + kb[q] * 4 * step + tok[q] * cpt * 32, step);
                if (lane < cpt) cs[kb[q] * NT * 8 + tok[q] * cpt + lane] = down;
            }
        }
    }
    __syncthreads();

    const uint32_t xs_a = smem_addr(smem), cs_a = smem_addr(cs) + t * 8;
    uint32_t x_lane[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) x_lane[nt] = xs_a + (min(nt * 8 + g, a.nc - 1) * 4 + t) * 16;
    float* park = reinterpret_cast<float*>(smem + a.park_off);
    float tot[NT][4] = {};
    int slot = 0, ls = n_k ? u0 / n_k : 0, kb = n_k ? u0 - ls * n_k : 0;
    for (int u = u0; u < u1; ++u) {
        cp_wait<kDepth - 1>();
        __syncwarp();
        const uint32_t at = ring + slot * a.unit_bytes;
        q4_unit<NT, SETS, ASYM>(tot, at, lane, a.bf16_scales != 0,
                                [&](int nt, int j) { return lds128(x_lane[nt] + (uint32_t)((kb * 4 + j) * step * 2)); },
                                [&](int nt) { return lds_f2(cs_a + (kb * NT + nt) * 32); });
        __syncwarp();
        fetch(at);
        if (++slot == kDepth) slot = 0;
        if (++kb == n_k || u + 1 == u1) {
            // piece (warp, strip) parks in slot warp + strip: along the units one of the two grows at every change
            float* p = park + (warp + ls) * 16 * a.nc + g * a.nc;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int c = nt * 8 + 2 * t + (i & 1);
                    if (c < a.nc) p[(i >> 1) * 8 * a.nc + c] = tot[nt][i];
                    tot[nt][i] = 0.0f;
                }
            }
            kb = 0;
            ++ls;
        }
    }
    cp_wait<0>();
    __syncthreads();

    // add the warps' pieces of every row in warp order; each CTA of the cluster finishes an equal part of the results
    const int rows = n_s * 16, outs = rows * a.tokens, share = (outs + S - 1) / S;
    float* red = reinterpret_cast<float*>(smem + a.red_off);
    if (S > 1) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");      // every CTA of the cluster has started
    for (int o = tid; o < outs; o += kThreads) {
        const int token = o / rows, r = o - token * rows, strip = r >> 4;
        float v = 0.0f;
        if (n_k) {
            const int w_lo = (int)(((int64_t)kWarps * (strip * n_k + 1) - 1) / U), w_hi = (int)(((int64_t)kWarps * (strip * n_k + n_k) - 1) / U);
            for (int w = w_lo; w <= w_hi; ++w) {
                if (U * w / kWarps == U * (w + 1) / kWarps) continue;
                const float* p = park + ((w + strip) * 16 + (r & 15)) * a.nc + token * cpt;
                v += cpt == 2 ? p[0] + p[1] : p[0];
            }
        }
        const int owner = o / share;
        if (S > 1) st_cluster(smem_addr(red + rank * share + (o - owner * share)), (uint32_t)owner, v);
        else red[o] = v;
    }
    if (S > 1) {
        asm volatile("barrier.cluster.arrive.release;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    }
    const int first = rank * share, last = min(outs, first + share);
    for (int o = first + tid; o < last; o += kThreads) {
        const int token = o / rows, m = s0 * 16 + o - token * rows;
        if (m >= a.M) continue;
        float v = 0.0f;
        for (int q = 0; q < S; ++q) v += red[q * share + o - first];
        if (a.bias) v += a.bias[m];
        if (a.act == PP_ACT_RELU) v = v > 0.0f || v != v ? v : 0.0f;
        store_y(a.y, (int64_t)token * a.ldy + m, a.y_type, v);
    }
}

using Kernel = void (*)(const Q4Args);
template <int NT, int SETS> Kernel pick_asym(bool asym) { return asym ? q4_kernel<NT, SETS, true> : q4_kernel<NT, SETS, false>; }
template <int NT> Kernel pick_sets(int sets, bool asym) {
    return sets == 4 ? pick_asym<NT, 4>(asym) : sets == 2 ? pick_asym<NT, 2>(asym) : pick_asym<NT, 1>(asym);
}
Kernel pick_kernel(int nt, int sets, bool asym) {
    return nt == 1 ? pick_sets<1>(sets, asym) : nt == 2 ? pick_sets<2>(sets, asym) : pick_sets<4>(sets, asym);
}

constexpr int kMaxSmem = 227 * 1024;

// Shared memory of a launch with clusters of S CTAs that own up to n_s strips each; fills in the offsets.
size_t plan_smem(Q4Args& a, int S, int n_s) {
    const int nt = a.nc <= 8 ? 1 : a.nc <= 16 ? 2 : 4, n_k = (a.blocks + S - 1) / S;
    size_t at = (size_t)n_k * kQ4UnitCols * a.nc * 2;
    a.cs_off = (int)at;
    at += (size_t)n_k * nt * 32;
    a.ring_off = (int)(at = (at + 127) / 128 * 128);
    at += (size_t)kWarps * kDepth * a.unit_bytes;
    a.park_off = (int)at;
    at += (size_t)(n_s + kWarps) * 16 * a.nc * 4;
    a.red_off = (int)at;
    const size_t outs = (size_t)n_s * 16 * a.tokens;
    at += (outs + S - 1) / S * S * 4;
    return at;
}

cudaError_t opt_in(const void* kernel) {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem);
}

// Rows of one strip and block to a unit: a thread writes the 16 bytes one lane of q4_unit reads.
__global__ void q4_pack_kernel(unsigned char* dst, const uint8_t* codes, const uint16_t* scales, const uint8_t* zeros, int rows, int cols,
                               int group, int groups, int strips, int blocks, int sets, int unit_bytes, int paired, int64_t n_units) {
    const int64_t stride = (int64_t)gridDim.x * blockDim.x;
    const int64_t code_ld = (cols + 1) / 2;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n_units * 64; i += stride) {
        const int64_t unit = i >> 6;
        const int part = (int)(i & 63), lane = part & 31, half = part >> 5, g = lane >> 2, t = lane & 3;
        const int block = (int)(unit % blocks);
        const int64_t ms = unit / blocks;                     // matrix * strips + strip
        const int strip = (int)(ms % strips);
        const int64_t row0 = ms / strips * rows;              // first row of the matrix among all rows
        unsigned char* u = dst + unit * unit_bytes;
        uint32_t w[4];
        for (int k = 0; k < 4; ++k) {
            const int c = block * kQ4UnitCols + 32 * (2 * half + k / 2) + 8 * t + 4 * (k & 1);
            w[k] = 0u;
            for (int h = 0; h < 2; ++h) {
                const int r = strip_row(rows, paired, strip, g, h);
                if (r < 0) continue;
                const uint8_t* p = codes + (row0 + r) * code_ld + c / 2;
                for (int e = 0; e < 4; ++e) {
                    if (c + e >= cols) break;
                    const uint32_t q = (p[e / 2] >> (4 * (e & 1))) & 15u;
                    w[k] |= q << (4 * h + 8 * (e / 2) + 16 * (e & 1));
                }
            }
        }
        *reinterpret_cast<uint4*>(u + half * 512 + lane * 16) = make_uint4(w[0], w[1], w[2], w[3]);
        if (part < sets * 16) {                               // entry 2 g + h of set part / 16: row g + 8 h
            const int set = part >> 4, e = part & 15, r = strip_row(rows, paired, strip, e >> 1, e & 1);
            const int col = block * kQ4UnitCols + set * (kQ4UnitCols / sets);
            const bool in = r >= 0 && col < cols;
            const int64_t at = in ? (row0 + r) * groups + (group ? col / group : 0) : 0;
            reinterpret_cast<uint16_t*>(u + 1024)[part] = in ? scales[at] : (uint16_t)0;
            if (zeros) u[1024 + sets * 32 + part] = in ? (uint8_t)((zeros[at] & 15u) << (4 * (e & 1))) : (uint8_t)0;
        }
    }
}

}  // namespace

cudaError_t launch_q4_pack(void* dst, const void* codes, const void* scales, const void* zeros, int count, int rows, int cols, int group,
                           bool paired, cudaStream_t stream) {
    const int strips = strips_of(rows, paired), blocks = (cols + kQ4UnitCols - 1) / kQ4UnitCols, sets = q4_sets(group);
    const int groups = group ? (cols + group - 1) / group : 1;
    const int64_t n = (int64_t)count * strips * blocks;
    const unsigned grid = (unsigned)std::min<int64_t>((n * 64 + 255) / 256, 148 * 32);
    q4_pack_kernel<<<grid, 256, 0, stream>>>(static_cast<unsigned char*>(dst), static_cast<const uint8_t*>(codes),
                                             static_cast<const uint16_t*>(scales), static_cast<const uint8_t*>(zeros), rows, cols, group, groups,
                                             strips, blocks, sets, q4_unit_bytes(sets, zeros != nullptr), paired, n);
    return cudaGetLastError();
}

}  // namespace pp

using namespace pp;

extern "C" pp_status_t pp_q4_destroy(pp_q4_t* L) {
    if (!L) return PP_ERR_INVALID_ARG;
    cudaFree(L->units);
    cudaFree(L->bias);
    delete L;
    return PP_OK;
}

extern "C" pp_status_t pp_q4_create(pp_q4_t** out, int M, int N, int group, const void* codes, const void* scales, pp_dtype_t scale_type,
                                    const void* zeros, const float* bias, void* cuda_stream) {
    if (!out) return PP_ERR_INVALID_ARG;
    *out = nullptr;
    if (M < 1 || N < 1 || !codes || !scales || group < 0 || !aligned_to(scales, 2) || !aligned_to(bias, 4)) return PP_ERR_INVALID_ARG;
    if (!is_16bit(scale_type) || !q4_group_ok(group) || M > (1 << 24) || N > (1 << 18)) return PP_ERR_UNSUPPORTED;
    pp_q4* L = new (std::nothrow) pp_q4{};
    if (!L) return PP_ERR_ALLOC;
    L->M = M;
    L->N = N;
    L->group = group;
    L->sets = q4_sets(group);
    L->strips = strips_of(M, false);
    L->blocks = (N + kQ4UnitCols - 1) / kQ4UnitCols;
    L->asym = zeros != nullptr;
    L->bf16_scales = scale_type == PP_BF16;
    const size_t bytes = (size_t)L->strips * L->blocks * q4_unit_bytes(L->sets, L->asym);
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    pp_status_t st = PP_OK;
    if ((cudaMalloc(&L->units, bytes) != cudaSuccess || (bias && cudaMalloc(&L->bias, (size_t)M * 4) != cudaSuccess))) {
        cudaGetLastError();
        st = PP_ERR_ALLOC;
    }
    if (st == PP_OK && (launch_q4_pack(L->units, codes, scales, zeros, 1, M, N, group, false, s) != cudaSuccess ||
                        (bias && cudaMemcpyAsync(L->bias, bias, (size_t)M * 4, cudaMemcpyDeviceToDevice, s) != cudaSuccess) ||
                        cudaStreamSynchronize(s) != cudaSuccess)) st = PP_ERR_CUDA;
    for (int nt = 1; nt <= 4 && st == PP_OK; nt *= 2)
        if (opt_in(reinterpret_cast<const void*>(pick_kernel(nt, L->sets, L->asym))) != cudaSuccess) st = PP_ERR_CUDA;
    // clusters resident at once, for a CTA of ordinary size (the GPCs hold different numbers of SMs)
    for (int S = 1; S <= 8 && st == PP_OK; S *= 2) {
        cudaLaunchAttribute at;
        at.id = cudaLaunchAttributeClusterDimension;
        at.val.clusterDim.x = (unsigned)S;
        at.val.clusterDim.y = at.val.clusterDim.z = 1;
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3(S);
        cfg.blockDim = dim3(kThreads);
        cfg.dynamicSmemBytes = 120 * 1024;      // one CTA to an SM
        cfg.attrs = &at;
        cfg.numAttrs = 1;
        int n = 0;
        if (cudaOccupancyMaxActiveClusters(&n, pick_kernel(1, L->sets, L->asym), &cfg) != cudaSuccess || n < 1) st = PP_ERR_CUDA;
        L->max_clusters[S] = n;
    }
    if (st != PP_OK) {
        pp_q4_destroy(L);
        return st;
    }
    *out = L;
    return PP_OK;
}

extern "C" pp_status_t pp_q4_launch_info(const pp_q4_t* L, int32_t out[4]) {
    if (!L || !out) return PP_ERR_INVALID_ARG;
    for (int i = 0; i < 4; ++i) out[i] = L->max_clusters[1 << i];
    return PP_OK;
}

extern "C" pp_status_t pp_q4_forward(pp_q4_t* L, const void* x, int64_t ldx, pp_dtype_t x_type, const float* x_scales, int x_group, void* y,
                                     pp_dtype_t y_type, int batch, pp_act_t act, void* cuda_stream) {
    if (!L || !x || !y || x == y || batch < 1 || (batch > 1 && ldx < L->N)) return PP_ERR_INVALID_ARG;
    if (act != PP_ACT_IDENTITY && act != PP_ACT_RELU) return PP_ERR_INVALID_ARG;
    if ((!is_float(x_type) && !is_8bit(x_type)) || !is_float(y_type)) return PP_ERR_UNSUPPORTED;
    if (is_8bit(x_type) ? !x_scales : x_scales != nullptr) return PP_ERR_INVALID_ARG;
    if (x_group != 0 && (!is_8bit(x_type) || x_group < 0 || x_group % kQ4UnitCols != 0)) return PP_ERR_UNSUPPORTED;
    const int xb = type_bytes(x_type), yb = type_bytes(y_type);
    if (!aligned_to(x, xb) || !aligned_to(y, yb) || !aligned_to(x_scales, 4)) return PP_ERR_INVALID_ARG;
    Q4Args a{};
    a.units = L->units;
    a.bias = L->bias;
    a.in.ld = ldx;
    a.in.type = x_type;
    a.in.scale_ld = x_group ? (L->N + x_group - 1) / x_group : 1;
    a.in.group_blocks = x_group / kQ4UnitCols;
    a.in.cols = L->N;
    a.in.vec = aligned_to(x, 4 * xb) && (batch == 1 || ldx % 4 == 0);
    a.ldy = L->M;
    a.y_type = y_type;
    a.act = act;
    a.M = L->M;
    a.strips = L->strips;
    a.blocks = L->blocks;
    a.unit_bytes = q4_unit_bytes(L->sets, L->asym);
    a.bf16_scales = L->bf16_scales;
    const int cpt = columns_per_token(x_type);
    int most = kMaxCols / cpt;                       // tokens of one launch
    for (int b0 = 0; b0 < batch;) {
        a.tokens = std::min(batch - b0, most);
        a.nc = a.tokens * cpt;
        a.in.x = static_cast<const char*>(x) + (int64_t)b0 * ldx * xb;
        a.in.scales = x_scales ? x_scales + (int64_t)b0 * a.in.scale_ld : nullptr;
        a.y = static_cast<char*>(y) + (int64_t)b0 * L->M * yb;
        // cluster size: the one whose busiest CTA has the fewest units
        int best = 0, best_n = 0;
        int64_t best_cost = 0;
        for (int S = 1; S <= 8; S *= 2) {
            const int n = std::max(std::min(L->strips, L->max_clusters[S]), (L->strips + kMaxStrips - 1) / kMaxStrips);
            const int n_s = (L->strips + n - 1) / n, n_k = (L->blocks + S - 1) / S;
            if (S > L->blocks || plan_smem(a, S, n_s) > (size_t)kMaxSmem) continue;
            const int64_t cost = (int64_t)n_s * n_k;
            if (!best || cost < best_cost) best = S, best_n = n, best_cost = cost;
        }
        if (!best) {                                 // x does not fit: fewer tokens at a time
            if (a.tokens == 1) return PP_ERR_UNSUPPORTED;
            most = a.tokens / 2;
            continue;
        }
        const size_t smem = plan_smem(a, best, (L->strips + best_n - 1) / best_n);
        const Kernel k = pick_kernel(a.nc <= 8 ? 1 : a.nc <= 16 ? 2 : 4, L->sets, L->asym);
        if (launch_pdl(k, dim3(best * best_n), dim3(kThreads), smem, static_cast<cudaStream_t>(cuda_stream), best, a) != cudaSuccess)
            return PP_ERR_CUDA;
        b0 += a.tokens;
    }
    return PP_OK;
}
