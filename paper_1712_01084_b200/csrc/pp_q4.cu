// y = act(W x + b) with 4-bit weights and group scales, for a few input vectors: layout (pp_q4.cuh), the kernel that
// rewrites plain codes into units, the product, and the C entry points.
//
// The product reads every weight once, so it is bound by HBM for large matrices and by the latency of one launch for
// small ones.  A cluster of S CTAs owns a run of 16-row strips; its CTAs own S equal parts of the columns, so each
// stages only its part of x.  A CTA's units, strip after strip, are dealt to its 16 warps in equal contiguous runs;
// every warp keeps a ring of units in flight in shared memory with 16-byte asynchronous copies, requested before the
// wait for the previous kernel (weights are never written by a kernel).  Partial sums meet in shared memory, those of
// the other CTAs arrive there through the cluster's distributed shared memory; all are added in one fixed order.
//
// Products, one or two vectors (eight of 8-bit integers): the integer tensor-core instruction (16 x 8 x 32, 8-bit operands,
// exact sums).  The codes need one mask instruction per four weights, where binary16 operands need 4.5.  x becomes fixed
// point: each block of 128 columns of a vector is multiplied by a power of two that brings its largest magnitude to
// (2^30, 0.996 * 2^31], rounded to whole numbers, and written as four signed bytes, one column of the product each: an
// error of at most 2^-31 of the block's largest element.  Eight columns cost what one costs, so the extra columns are free.
// (Three bytes would do for blocks of even elements; beside an element 10^4 times as large, in rows whose weight is 0
// there, they err by several times an fp32 sum's 10^-5.)  8-bit integers are one column, e4m3 values times 2^9 whole numbers
// of three bytes; both are exact.
//   sum (q - z) d = sum q d - z sum d  over each set of scales, in exact integers (sum d is made while x is staged and
// the product starts from -z sum d); then one fp32 multiply-add per set with (scale of the row) * (scale of the column).
// More vectors: binary16 products (16 x 8 x 16, fp32 sums), where a vector takes one column, an f32 vector two (the second
// holds what the first one's 11 bits leave over); bf16 and f32 blocks of 128 columns are brought to [2^13, 2^14) by a power
// of two first.  Eight vectors would be 32 columns of bytes.
//
// 8192 x 8192, us in a graph: one vector 9.8 (3.5 TB/s), two 10.8, four of bf16 11.5, eight 13.4, sixteen 16.9, sixteen of f32
// 23.5 (there a unit costs 256 cycles of matrix instructions and 300 of shared memory); int8 9.2, eight vectors 13.3; e4m3 9.5,
// 13.4; every 16 vectors more the same again.  4096 x 4096, one vector, 4.7.
#include "pp_q4.cuh"

#include <algorithm>
#include <new>

struct pp_q4 {
    int M, N, group, sets, strips, blocks;
    bool asym, bf16_scales;
    unsigned char *units, *sets_at;   // codes and sets of the units
    float* bias;
    int max_clusters[9];      // clusters of this size that the device holds at once
};

namespace pp {
namespace {

constexpr int kWarps = 16, kThreads = kWarps * 32, kMaxStrips = 64, kMaxTokens = 16;
constexpr int kParkLd = 20;           // floats between parked columns of 16 rows: a warp's 32 values hit 32 banks
// Units each warp keeps in flight: 4 (70 KB an SM) keep HBM busy; 7 where x is small, so that more of the next call's weights
// are on their way during this one's end; with 32 columns there is room for 3.  (7 also leave room for one CTA to an SM
// only.  With two, the next call's CTAs start beside this one's; 8192 x 8192 then took 8.7 us a call, but 12 us whenever
// the CTAs of a call land on one SM twice, which lasts until the stream runs dry.  One took 9.3 us, always.)
__host__ __device__ constexpr int depth_of(int nt) { return nt == 4 ? 3 : nt == 1 ? 7 : 4; }
constexpr int kShallow = 4;           // of binary16 products with one tile, where x leaves no room for 7
// Columns of the product a vector takes.
__host__ __device__ constexpr int columns_of(bool bytes, int xtype) { return bytes ? (xtype == PP_I8 ? 1 : xtype == PP_E4M3 ? 3 : 4) : xtype == PP_F32 ? 2 : 1; }
bool as_bytes(int tokens, int xtype) { return tokens * columns_of(true, xtype) <= 8; }
// (16 vectors to a launch: 32 of bf16 in one, four tiles, took 53 us, in two launches 34 us; 8192 x 8192)
int tiles_of(int nc) { return nc <= 8 ? 1 : nc <= 16 ? 2 : 4; }

struct Q4Args {
    const unsigned char *units, *sets;
    const float* bias;
    XIn in;
    void* y;
    int y_type, act, tokens, nc;          // nc: columns of the staged input
    int y_vec;                            // four results of a vector lie in one access
    int M, blocks, slot_bytes, bf16_scales;
    int strips_each, strips_more;         // a cluster has strips_each strips, the first strips_more of them one more
    int blocks_each, blocks_more;         // the same for a CTA of a cluster and the blocks of the columns
    int plan_off, ring_off, cs_off, sum_off, park_off, red_off;      // shared memory; the staged input is at 0
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
template <typename V> __device__ __forceinline__ void st_cluster(uint32_t local, uint32_t rank, const V& v) {     // 1 or 4 floats
    uint32_t remote;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(local), "r"(rank));
    if constexpr (sizeof(V) == 4) asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(remote), "f"(v.v[0]) : "memory");
    else asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(remote), "f"(v.v[0]), "f"(v.v[1]), "f"(v.v[2]), "f"(v.v[3]) : "memory");
}

// N results from i on, the first n of them; in one access where vec says so.
template <typename T, int N> __device__ __forceinline__ void store_as(T* y, const Pack<float, N>& v, int n, bool vec) {
    Pack<T, N> p;
#pragma unroll
    for (int i = 0; i < N; ++i) p.v[i] = from_float<T>(v.v[i]);
    if (vec) {
        *reinterpret_cast<Pack<T, N>*>(y) = p;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < n) y[i] = p.v[i];
    }
}
template <int N> __device__ __forceinline__ void store_y(void* y, int64_t i, int type, const Pack<float, N>& v, int n, bool vec) {
    if (type == PP_F32) store_as(static_cast<float*>(y) + i, v, n, vec);
    else if (type == PP_F16) store_as(static_cast<__half*>(y) + i, v, n, vec);
    else store_as(static_cast<__nv_bfloat16*>(y) + i, v, n, vec);
}

// A warp's block of 128 columns of one vector in binary16, four per lane, columns 4i + 1 and 4i + 2 exchanged; rest: what
// f32 leaves over.  The result is the power of two to multiply with.
template <typename T> __device__ __forceinline__ float halves(const Pack<T, 4>& x, uint2& h, uint2& rest) {
    float f[4], down = 1.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = to_float(x.v[i]);
    if constexpr (std::is_same_v<T, float> || std::is_same_v<T, __nv_bfloat16>) {
        uint32_t most = 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i) most = max(most, __float_as_uint(f[i]) & 0x7fffffffu);
        float up;
        f16_scale(__uint_as_float(__reduce_max_sync(0xffffffffu, most)), up, down);
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] *= up;
    }
    const __half2 a = __floats2half2_rn(f[0], f[2]), b = __floats2half2_rn(f[1], f[3]);
    h = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
    if constexpr (std::is_same_v<T, float>) {
        const float2 p = __half22float2(a), q = __half22float2(b);
        const __half2 c = __floats2half2_rn(f[0] - p.x, f[2] - p.y), d = __floats2half2_rn(f[1] - q.x, f[3] - q.y);
        rest = make_uint2(*reinterpret_cast<const uint32_t*>(&c), *reinterpret_cast<const uint32_t*>(&d));
    }
    return down;
}

// This CTA's columns of x and, per block of 128 columns, what a column stands for (cs) and its sum over each set of scales
// (sums, bytes only).  Bytes are laid out [64 columns][column of the product][lane t][8 bytes of 32 columns, 8 of the next],
// halves [32 columns][column of the product][lane t][8 halves]: what a lane reads at once.  Several blocks of four elements
// per lane are requested before the first is converted, as a step of this loop is a trip to memory (two where a warp has two).
// then(): called once the first of them are on their way.
template <typename T, bool VEC, bool BYTES, int NT, int SETS, typename Then>
__device__ __forceinline__ void stage_rows(const Q4Args& a, unsigned char* xs, float* cs, int* sums, int k0, int n_k, int warp, int lane, Then then) {
    constexpr int kAhead = !VEC ? 1 : BYTES ? 2 : sizeof(T) == 4 ? 4 : 8;
    constexpr int cpt = BYTES ? byte_columns<T>() : std::is_same_v<T, float> ? 2 : 1;
    const int items = a.tokens * n_k, step = a.nc * 64;
    const Divider by_blocks(n_k);
    if (warp >= items) then();
    for (int base = warp; base < items; base += kAhead * kWarps) {
        Pack<T, 4> v[kAhead];
        float own[kAhead];
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            const int item = min(base + q * kWarps, items - 1), token = by_blocks.div(item), block = k0 + item - token * n_k;
            v[q] = load_four<VEC>(static_cast<const T*>(a.in.x) + token * a.in.ld, block * kQ4UnitCols + lane * 4, a.in.cols);
            if (sizeof(T) == 1) own[q] = a.in.scales[(int64_t)token * a.in.scale_ld + (a.in.group_blocks ? block / a.in.group_blocks : 0)];
        }
        if (base == warp) then();
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            const int item = base + q * kWarps, token = by_blocks.div(item), kb = item - token * n_k;
            if (item >= items) break;
            if constexpr (BYTES) {
                uint32_t w[cpt];
                float down;
                fixed_point(v[q], own[q], w, down);
                unsigned char* at = xs + (kb * 2 + (lane >> 4)) * step + token * cpt * 64 + ((lane >> 1) & 3) * 16 + (lane & 8) + (lane & 1) * 4;
#pragma unroll
                for (int c = 0; c < cpt; ++c) *reinterpret_cast<uint32_t*>(at + c * 64) = w[c];
                const int sum = byte_sums<SETS>(w, lane);
                constexpr int kLanes = 32 / SETS;            // of a set
                const int c = lane & (kLanes - 1), col = token * cpt + c;
                if (c < cpt) {
                    sums[(kb * SETS + lane / kLanes) * NT * 8 + col] = sum;
                    if (lane < cpt) cs[kb * NT * 8 + col] = down * byte_weight<cpt>(c);
                }
            } else {
                uint2 h, rest;
                const float down = halves(v[q], h, rest);
                unsigned char* at = xs + (kb * 4 + (lane >> 3)) * step + token * cpt * 64 + (lane & 7) * 8;
                *reinterpret_cast<uint2*>(at) = h;
                if (cpt == 2) *reinterpret_cast<uint2*>(at + 64) = rest;
                if (lane < cpt) cs[kb * NT * 8 + token * cpt + lane] = sizeof(T) == 1 ? own[q] : down;
            }
        }
    }
}

template <typename T, bool BYTES, int NT, int SETS, typename Then>
__device__ __forceinline__ void stage_x(const Q4Args& a, unsigned char* xs, float* cs, int* sums, int k0, int n_k, int warp, int lane, Then then) {
    if (a.in.vec) stage_rows<T, true, BYTES, NT, SETS>(a, xs, cs, sums, k0, n_k, warp, lane, then);
    else stage_rows<T, false, BYTES, NT, SETS>(a, xs, cs, sums, k0, n_k, warp, lane, then);
}

// (64 registers a thread with bytes: 8192 x 8192 takes 9.7 us, with the 70 to 80 that it would use 9.95)
template <bool BYTES, int NT, int SETS, bool ASYM, int DEPTH>
__global__ void __launch_bounds__(kThreads, BYTES ? 2 : 1) q4_kernel(const Q4Args a) {
    extern __shared__ __align__(128) unsigned char smem[];
    constexpr int kDepth = DEPTH;
    const int S = (int)cluster_size(), rank = (int)cluster_rank(), cl = S == 1 ? blockIdx.x : blockIdx.x / S;
    const int s0 = cl * a.strips_each + min(cl, a.strips_more), n_s = a.strips_each + (cl < a.strips_more);
    const int k0 = rank * a.blocks_each + min(rank, a.blocks_more), n_k = a.blocks_each + (rank < a.blocks_more);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int U = n_s * n_k, u0 = U * warp / kWarps, u1 = U * (warp + 1) / kWarps;
    if (S > 1) asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");

    // the first units of this warp: nothing in them depends on an earlier kernel
    const int ls0 = Divider(n_k).div(u0), kb0 = u0 - ls0 * n_k;
    constexpr int kSetBytes = SETS * (ASYM ? 48 : 32);
    unsigned char *const ring = smem + a.ring_off + warp * kDepth * a.slot_bytes, *const ring_end = ring + kDepth * a.slot_bytes;
    const int64_t at0 = (int64_t)(s0 + ls0) * a.blocks + k0 + kb0;
    const unsigned char *unit = a.units + at0 * kQ4CodeBytes + lane * 16, *sets = a.sets + at0 * kSetBytes + lane * 16;
    int todo = u1 - u0, run = n_k - kb0;                     // units still to request, and those of them in this strip
    auto fetch = [&](uint32_t slot) {
        if (todo > 0) {
            --todo;
            cp_async16(slot, unit);
            cp_async16(slot + 512, unit + 512);
            if (lane < kSetBytes / 16) cp_async16(slot + 1024, sets);
            unit += kQ4CodeBytes;
            sets += kSetBytes;
            if (--run == 0) {
                run = n_k;
                unit += (int64_t)(a.blocks - n_k) * kQ4CodeBytes;
                sets += (int64_t)(a.blocks - n_k) * kSetBytes;
            }
        }
        cp_commit();
    };
    // (with more vectors the rest of the ring is requested behind x, which it would hold back: 4096 x 9216, eight vectors,
    // 12.6 us for all of it before x, 10.2 for two; 8192 x 8192, sixteen f32 vectors, 25.2 and 23.5.  One vector is small
    // and loses by it: 4096 x 4096 5.7 -> 5.9 us)
    constexpr int kEarly = BYTES ? kDepth : 2;
#pragma unroll
    for (int d = 0; d < kEarly; ++d) fetch(smem_addr(ring) + d * a.slot_bytes + lane * 16);
    // which warps have units of each strip: half a warp looks at one
    uint16_t* plan = reinterpret_cast<uint16_t*>(smem + a.plan_off);
    for (int base = 0; base < n_s; base += kThreads / 16) {
        const int strip = base + (tid >> 4), w = tid & 15;
        const bool has = strip < n_s && max(U * w / kWarps, strip * n_k) < min(U * (w + 1) / kWarps, (strip + 1) * n_k);
        const uint32_t mask = __ballot_sync(0xffffffffu, has) >> (lane & 16);
        if (w == 0 && strip < n_s) plan[strip] = (uint16_t)mask;
    }

    pdl_wait();
    pdl_release();                       // not before the previous call has ended: the one after this must not run ahead of both
    float* cs = reinterpret_cast<float*>(smem + a.cs_off);
    int* sums = reinterpret_cast<int*>(smem + a.sum_off);
    const auto rest = [&] {
#pragma unroll
        for (int d = kEarly; d < kDepth; ++d) fetch(smem_addr(ring) + d * a.slot_bytes + lane * 16);
    };
    switch (a.in.type) {
        case PP_F32: stage_x<float, BYTES, NT, SETS>(a, smem, cs, sums, k0, n_k, warp, lane, rest); break;
        case PP_F16: stage_x<__half, BYTES, NT, SETS>(a, smem, cs, sums, k0, n_k, warp, lane, rest); break;
        case PP_BF16: stage_x<__nv_bfloat16, BYTES, NT, SETS>(a, smem, cs, sums, k0, n_k, warp, lane, rest); break;
        case PP_I8: stage_x<int8_t, BYTES, NT, SETS>(a, smem, cs, sums, k0, n_k, warp, lane, rest); break;
        default: stage_x<__nv_fp8_e4m3, BYTES, NT, SETS>(a, smem, cs, sums, k0, n_k, warp, lane, rest);
    }
    __syncthreads();

    const bool paired = !BYTES && a.nc != a.tokens;          // f32 in halves: a vector's two columns are neighbours in one lane
    const int parked = paired ? a.tokens : a.nc;             // columns that are parked
    const int step = a.nc * 64;                              // bytes to the next 64 columns of bytes, 32 columns of halves
    constexpr int kSteps = BYTES ? 2 : 4;                    // of a unit
    int x_lane[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) x_lane[nt] = (min(nt * 8 + g, a.nc - 1) * 4 + t) * 16;       // columns past the last repeat it
    float* park = reinterpret_cast<float*>(smem + a.park_off);
    float tot[NT][4] = {};
    unsigned char* at = ring;
    int ls = ls0, kb = kb0;
    for (int left = u1 - u0; left > 0; ++ls, kb = 0) {
        int n = min(n_k - kb, left);
        left -= n;
        const unsigned char* x = smem + kb * kSteps * step;
        const int* sum = sums + kb * SETS * NT * 8 + t * 2;
        const float* c = cs + kb * NT * 8 + t * 2;
        do {
            cp_wait<kDepth - 1>();
            __syncwarp();
            if constexpr (BYTES) {
                q4_unit_i8<NT, SETS, ASYM>(tot, at, lane, a.bf16_scales != 0,
                                           [&](int nt, int h) { return *reinterpret_cast<const uint4*>(x + h * step + x_lane[nt]); },
                                           [&](int nt, int set) { return *reinterpret_cast<const int2*>(sum + (set * NT + nt) * 8); },
                                           [&](int nt) { return *reinterpret_cast<const float2*>(c + nt * 8); });
            } else {
                q4_unit_f16<NT, SETS, ASYM>(tot, at, lane, a.bf16_scales != 0,
                                            [&](int nt, int j) { return *reinterpret_cast<const uint4*>(x + j * step + x_lane[nt]); },
                                            [&](int nt) { return *reinterpret_cast<const float2*>(c + nt * 8); });
            }
            __syncwarp();
            fetch(smem_addr(at) + lane * 16);
            at += a.slot_bytes;
            if (at == ring_end) at = ring;
            x += kSteps * step;
            sum += SETS * NT * 8;
            c += NT * 8;
        } while (--n);
        // piece (warp, strip) parks in slot warp + strip: along the units one of the two grows at every change
        float* p = park + (warp + ls) * kParkLd * parked + g;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int col = nt * 8 + 2 * t;
                if (paired) {
                    if (col < a.nc) p[col / 2 * kParkLd + h * 8] = tot[nt][2 * h] + tot[nt][2 * h + 1];
                } else {
                    if (col < parked) p[col * kParkLd + h * 8] = tot[nt][2 * h];
                    if (col + 1 < parked) p[(col + 1) * kParkLd + h * 8] = tot[nt][2 * h + 1];
                }
                tot[nt][2 * h] = tot[nt][2 * h + 1] = 0.0f;
            }
        }
    }
    cp_wait<0>();
    __syncthreads();

    // add the warps' pieces of every row in warp order; each CTA of the cluster finishes an equal part of the results.  With
    // more vectors a thread has four rows (8192 x 8192, sixteen f32 vectors: one row 29.0 us a call, four 25.5); one vector leaves most
    // threads without a row then (4096 x 4096: 4.9 and 5.3 us).
    constexpr int kRows = BYTES ? 1 : 4;
    using Rows = Pack<float, kRows>;
    const int per_token = n_s * (16 / kRows), outs = per_token * a.tokens, share = S == 1 ? outs : (outs + S - 1) / S;
    const int first = rank * share, last = min(outs, first + share);
    const int cpt = !BYTES || a.in.type == PP_I8 ? 1 : a.in.type == PP_E4M3 ? 3 : 4;     // parked columns of a vector
    const Divider by_token(per_token), by_share(share);
    Rows* red = reinterpret_cast<Rows*>(smem + a.red_off);
    Rows bias{};                                             // of this thread's first results: on their way during the barrier
    const auto row_of = [&](int o) { return s0 * 16 + (o - by_token.div(o) * per_token) * kRows; };
    const auto load_bias = [&](int m) {
#pragma unroll
        for (int i = 0; i < kRows; ++i)
            if (m + i < a.M) bias.v[i] = __ldg(a.bias + m + i);
    };
    if (a.bias && first + tid < last) load_bias(row_of(first + tid));
    if (S > 1) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");      // every CTA of the cluster has started
    for (int o = tid; o < outs; o += kThreads) {
        const int token = by_token.div(o), r = (o - token * per_token) * kRows, strip = r >> 4;
        Rows v{};
        for (uint32_t m = plan[strip]; m; m &= m - 1) {
            const float* p = park + (__ffs((int)m) - 1 + strip) * kParkLd * parked + token * cpt * kParkLd + (r & 15);
            Rows w = *reinterpret_cast<const Rows*>(p);
            if (BYTES && cpt > 1) w.v[0] += p[kParkLd] + (cpt == 4 ? p[2 * kParkLd] + p[3 * kParkLd] : p[2 * kParkLd]);
#pragma unroll
            for (int i = 0; i < kRows; ++i) v.v[i] += w.v[i];
        }
        if (S > 1) {
            const int owner = by_share.div(o);
            st_cluster(smem_addr(red + rank * share + o - owner * share), (uint32_t)owner, v);
        } else {
            red[o] = v;
        }
    }
    if (S > 1) {
        asm volatile("barrier.cluster.arrive.release;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    }
    for (int o = first + tid; o < last; o += kThreads) {
        const int token = by_token.div(o), m = row_of(o);
        if (m >= a.M) continue;
        Rows v{};
        for (int q = 0; q < S; ++q) {
            const Rows w = red[q * share + o - first];
#pragma unroll
            for (int i = 0; i < kRows; ++i) v.v[i] += w.v[i];
        }
        if (a.bias && o != first + tid) load_bias(m);
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            if (a.bias) v.v[i] += bias.v[i];
            if (a.act == PP_ACT_RELU) v.v[i] = v.v[i] > 0.0f || v.v[i] != v.v[i] ? v.v[i] : 0.0f;
        }
        store_y(a.y, (int64_t)token * a.M + m, a.y_type, v, a.M - m, kRows == 1 || a.y_vec);
    }
}

// How a launch multiplies: whole numbers or binary16, and units that each warp keeps in flight.
struct Form { bool bytes; int depth; };

using Kernel = void (*)(const Q4Args);
template <bool BYTES, int NT, int SETS, int DEPTH> Kernel pick_asym(bool asym) {
    return asym ? q4_kernel<BYTES, NT, SETS, true, DEPTH> : q4_kernel<BYTES, NT, SETS, false, DEPTH>;
}
template <bool BYTES, int NT, int DEPTH = depth_of(NT)> Kernel pick_sets(int sets, bool asym) {
    return sets == 4 ? pick_asym<BYTES, NT, 4, DEPTH>(asym) : sets == 2 ? pick_asym<BYTES, NT, 2, DEPTH>(asym) : pick_asym<BYTES, NT, 1, DEPTH>(asym);
}
Kernel pick_kernel(Form f, int nt, int sets, bool asym) {
    return f.bytes ? pick_sets<true, 1>(sets, asym) : nt == 4 ? pick_sets<false, 4>(sets, asym) : nt == 2 ? pick_sets<false, 2>(sets, asym)
         : f.depth == kShallow ? pick_sets<false, 1, kShallow>(sets, asym) : pick_sets<false, 1>(sets, asym);
}

constexpr int kMaxSmem = 227 * 1024;

// Shared memory of a launch with clusters of S CTAs that own up to n_s strips each; fills in the offsets.
size_t plan_smem(Q4Args& a, Form f, int sets, int S, int n_s) {
    const bool bytes = f.bytes;
    const int nt = tiles_of(a.nc), n_k = (a.blocks + S - 1) / S;
    size_t at = (size_t)n_k * kQ4UnitCols * a.nc * (bytes ? 1 : 2);
    a.cs_off = (int)at;
    at += (size_t)n_k * nt * 32;
    a.sum_off = (int)at;
    if (bytes) at += (size_t)n_k * sets * nt * 32;
    a.plan_off = (int)at;
    at += (size_t)n_s * 2;
    a.ring_off = (int)(at = (at + 127) / 128 * 128);
    at += (size_t)kWarps * f.depth * a.slot_bytes;
    a.park_off = (int)at;
    const bool paired = !bytes && a.nc != a.tokens;
    at += (size_t)(n_s + kWarps) * kParkLd * (paired ? a.tokens : a.nc) * 4;
    a.red_off = (int)at;
    const size_t row = bytes ? 1 : 4, outs = (size_t)n_s * 16 / row * a.tokens;       // rows to a thread
    at += (outs + S - 1) / S * S * row * 4;
    return at;
}

cudaError_t opt_in(const void* kernel) {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem);
}

// Rows of one strip and block to a unit: a thread writes the 16 bytes one lane of a product reads.
__global__ void q4_pack_kernel(unsigned char* dst, unsigned char* dst_sets, const uint8_t* codes, const uint16_t* scales, const uint8_t* zeros, int rows, int cols,
                               int group, int groups, int strips, int blocks, int sets, int set_bytes, int paired, int64_t n_units) {
    const int64_t stride = (int64_t)gridDim.x * blockDim.x;
    const int64_t code_ld = (cols + 1) / 2;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n_units * 64; i += stride) {
        const int64_t unit = i >> 6;
        const int part = (int)(i & 63), lane = part & 31, half = part >> 5, g = lane >> 2, t = lane & 3;
        const int block = (int)(unit % blocks);
        const int64_t ms = unit / blocks;                     // matrix * strips + strip
        const int strip = (int)(ms % strips);
        const int64_t row0 = ms / strips * rows;              // first row of the matrix among all rows
        uint32_t w[4];
        for (int k = 0; k < 4; ++k) {
            const int c = block * kQ4UnitCols + 32 * (2 * half + k / 2) + 8 * t + 4 * (k & 1);      // the word's four columns
            w[k] = 0u;
            for (int h = 0; h < 2; ++h) {
                const int r = strip_row(rows, paired, strip, g, h);
                if (r < 0) continue;
                const uint8_t* p = codes + (row0 + r) * code_ld + c / 2;
                for (int e = 0; e < 4; ++e) {
                    if (c + e >= cols) break;
                    const uint32_t q = (p[e / 2] >> (4 * (e & 1))) & 15u;
                    w[k] |= q << (8 * e + 4 * h);
                }
            }
        }
        *reinterpret_cast<uint4*>(dst + unit * kQ4CodeBytes + half * 512 + lane * 16) = make_uint4(w[0], w[1], w[2], w[3]);
        if (part < sets * 16) {                               // entry 2 g + h of set part / 16: row g + 8 h
            const int set = part >> 4, e = part & 15, r = strip_row(rows, paired, strip, e >> 1, e & 1);
            const int col = block * kQ4UnitCols + set * (kQ4UnitCols / sets);
            const bool in = r >= 0 && col < cols;
            const int64_t at = in ? (row0 + r) * groups + (group ? col / group : 0) : 0;
            unsigned char* u = dst_sets + unit * set_bytes;
            reinterpret_cast<uint16_t*>(u)[part] = in ? scales[at] : (uint16_t)0;
            if (zeros) u[sets * 32 + part] = in ? (uint8_t)((zeros[at] & 15u) << (4 * (e & 1))) : (uint8_t)0;
        }
    }
}

}  // namespace

cudaError_t launch_q4_pack(void* dst, void* dst_sets, const void* codes, const void* scales, const void* zeros, int count, int rows, int cols, int group,
                           bool paired, cudaStream_t stream) {
    const int strips = strips_of(rows, paired), blocks = (cols + kQ4UnitCols - 1) / kQ4UnitCols, sets = q4_sets(group);
    const int groups = group ? (cols + group - 1) / group : 1;
    const int64_t n = (int64_t)count * strips * blocks;
    const unsigned grid = (unsigned)std::min<int64_t>((n * 64 + 255) / 256, sm_count() * 32);
    q4_pack_kernel<<<grid, 256, 0, stream>>>(static_cast<unsigned char*>(dst), static_cast<unsigned char*>(dst_sets), static_cast<const uint8_t*>(codes),
                                             static_cast<const uint16_t*>(scales), static_cast<const uint8_t*>(zeros), rows, cols, group, groups,
                                             strips, blocks, sets, q4_set_bytes(sets, zeros != nullptr), paired, n);
    return cudaGetLastError();
}

}  // namespace pp

using namespace pp;

extern "C" pp_status_t pp_q4_destroy(pp_q4_t* L) {
    if (!L) return PP_ERR_INVALID_ARG;
    cudaFree(L->units);
    cudaFree(L->sets_at);
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
    const size_t units = (size_t)L->strips * L->blocks;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    pp_status_t st = PP_OK;
    if ((cudaMalloc(&L->units, units * kQ4CodeBytes) != cudaSuccess ||
         cudaMalloc(&L->sets_at, units * q4_set_bytes(L->sets, L->asym)) != cudaSuccess || (bias && cudaMalloc(&L->bias, (size_t)M * 4) != cudaSuccess))) {
        st = PP_ERR_ALLOC;
    }
    if (st == PP_OK && (launch_q4_pack(L->units, L->sets_at, codes, scales, zeros, 1, M, N, group, false, s) != cudaSuccess ||
                        (bias && cudaMemcpyAsync(L->bias, bias, (size_t)M * 4, cudaMemcpyDeviceToDevice, s) != cudaSuccess) ||
                        cudaStreamSynchronize(s) != cudaSuccess)) st = PP_ERR_CUDA;
    for (const Kernel k : {pick_kernel({true, 0}, 1, L->sets, L->asym), pick_kernel({false, kShallow}, 1, L->sets, L->asym),
                           pick_kernel({false, 0}, 1, L->sets, L->asym), pick_kernel({false, 0}, 2, L->sets, L->asym),
                           pick_kernel({false, 0}, 4, L->sets, L->asym)})
        if (st == PP_OK && opt_in(reinterpret_cast<const void*>(k)) != cudaSuccess) st = PP_ERR_CUDA;
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
        if (cudaOccupancyMaxActiveClusters(&n, pick_kernel({true, 0}, 1, L->sets, L->asym), &cfg) != cudaSuccess || n < 1) st = PP_ERR_CUDA;
        L->max_clusters[S] = n;
    }
    if (st != PP_OK) {
        cudaGetLastError();
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
    if (!L || !x || !y || batch < 1 || (batch > 1 && ldx < L->N)) return PP_ERR_INVALID_ARG;
    if (act != PP_ACT_IDENTITY && act != PP_ACT_RELU) return PP_ERR_INVALID_ARG;
    if ((!is_float(x_type) && !is_8bit(x_type)) || !is_float(y_type)) return PP_ERR_UNSUPPORTED;
    if (is_8bit(x_type) ? !x_scales : x_scales != nullptr) return PP_ERR_INVALID_ARG;
    if (x_group != 0 && (!is_8bit(x_type) || x_group < 0 || x_group % kQ4UnitCols != 0)) return PP_ERR_UNSUPPORTED;
    const int xb = type_bytes(x_type), yb = type_bytes(y_type);
    if (!aligned_to(x, xb) || !aligned_to(y, yb) || !aligned_to(x_scales, 4)) return PP_ERR_INVALID_ARG;
    const int64_t y_bytes = (int64_t)batch * L->M * yb;
    const int64_t scales_bytes = (int64_t)batch * (x_group ? (L->N + x_group - 1) / x_group : 1) * 4;
    if (share_bytes(x, (int64_t)L->N * xb, ldx * xb, batch, y, y_bytes, y_bytes, 1) ||
        share_bytes(x_scales, scales_bytes, scales_bytes, 1, y, y_bytes, y_bytes, 1)) return PP_ERR_INVALID_ARG;
    Q4Args a{};
    a.units = L->units;
    a.bias = L->bias;
    a.in.ld = ldx;
    a.in.type = x_type;
    a.in.scale_ld = x_group ? (L->N + x_group - 1) / x_group : 1;
    a.in.group_blocks = x_group / kQ4UnitCols;
    a.in.cols = L->N;
    a.in.vec = aligned_to(x, 4 * xb) && (batch == 1 || ldx % 4 == 0) && L->N % 4 == 0;
    a.y_type = y_type;
    a.act = act;
    a.M = L->M;
    a.blocks = L->blocks;
    a.sets = L->sets_at;
    a.slot_bytes = kQ4CodeBytes + (q4_set_bytes(L->sets, L->asym) + 127) / 128 * 128;      // slots start on 128 bytes
    a.bf16_scales = L->bf16_scales;
    int most = kMaxTokens;                       // tokens of one launch
    for (int b0 = 0; b0 < batch;) {
        a.tokens = std::min(batch - b0, most);
        a.in.x = static_cast<const char*>(x) + (int64_t)b0 * ldx * xb;
        a.in.scales = x_scales ? x_scales + (int64_t)b0 * a.in.scale_ld : nullptr;
        a.y = static_cast<char*>(y) + (int64_t)b0 * L->M * yb;
        a.y_vec = L->M % 4 == 0 && aligned_to(a.y, 4 * yb);
        // cluster size and strips to a cluster: the fewest units on the busiest SM, counting what staging a block of a
        // token's columns costs as half a unit.  More strips than one round of clusters can hold go in several rounds.
        int best = 0, best_n = 0;
        int64_t best_cost = 0;
        Form form{};
        const auto plan = [&](Form f) {
            form = f;
            a.nc = a.tokens * columns_of(f.bytes, x_type);
            for (int S = 1; S <= 8 && S <= L->blocks; S *= 2) {
                const int n_k = (L->blocks + S - 1) / S;
                for (int rounds = 1; rounds <= L->strips; ++rounds) {
                    const int n = std::min(L->strips, L->max_clusters[S] * rounds), n_s = (L->strips + n - 1) / n;
                    if (n_s > kMaxStrips || plan_smem(a, f, L->sets, S, n_s) > (size_t)kMaxSmem) {
                        if (n_s == 1) break;
                        continue;
                    }
                    const int64_t cost = rounds * (2ll * n_s + a.tokens) * n_k;
                    if (!best || cost < best_cost) best = S, best_n = n, best_cost = cost;
                    break;
                }
            }
            return best != 0;
        };
        // bytes, where they are the faster form and fit (a float vector of up to some 120,000 columns); then binary16, a shorter
        // ring before fewer vectors, as fewer vectors read the weights again
        const int nt = tiles_of(a.tokens * columns_of(false, x_type));
        if (!(as_bytes(a.tokens, x_type) && plan({true, depth_of(1)})) && !plan({false, depth_of(nt)}) && nt == 1) plan({false, kShallow});
        if (!best) {                                 // x does not fit: fewer tokens at a time (one does, up to the 2^18 columns of a layer)
            if (a.tokens == 1) return PP_ERR_UNSUPPORTED;
            most = a.tokens / 2;
            continue;
        }
        const size_t smem = plan_smem(a, form, L->sets, best, (L->strips + best_n - 1) / best_n);
        a.strips_each = L->strips / best_n;
        a.strips_more = L->strips % best_n;
        a.blocks_each = L->blocks / best;
        a.blocks_more = L->blocks % best;
        const Kernel k = pick_kernel(form, tiles_of(a.nc), L->sets, L->asym);
        const pp_status_t st = status_of(launch_pdl(k, dim3(best * best_n), dim3(kThreads), smem, static_cast<cudaStream_t>(cuda_stream), best, a));
        if (st != PP_OK) return st;
        b0 += a.tokens;
    }
    return PP_OK;
}
