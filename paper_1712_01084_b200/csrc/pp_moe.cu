// A whole mixture-of-experts layer for a few tokens in one cooperative kernel.
//
//   l = R x (fp32),  the top_k largest (ties: the lowest index),  p = softmax(l), renormalised over the chosen or not
//   y = sum_j D_e(j) ( p_j * silu(G_e(j) x) * (U_e(j) x) )
//
// With a few tokens every chosen expert's weights are read once for one to a few columns, so the layer is bound by HBM
// on those weights, and for one token by the three steps that wait for one another:
//   step 0  the first CTAs turn the tokens into columns of the products' type, every warp of the grid takes (token,
//           expert) pairs of the router;                                                     -- grid barrier --
//   step 1  every CTA chooses the experts for itself (a warp per token; no second barrier) and lists those that some token
//           chose; the grid streams their gate and up rows, eight rows of each to a strip, so
//           whoever finishes a strip has both halves of act = p silu(g) u;                   -- grid barrier --
//   step 2  the grid streams the down rows; a strip of 16 rows of y collects all experts.  The first of these weights are
//           requested before the barrier.
// In steps 1 and 2 all units (1 KB of weights) form one sequence that is cut into equal parts, one per CTA, wherever that
// falls; inside a CTA a round of strips is dealt to the 16 warps in equal runs, each with a ring of asynchronous copies in
// flight.  Warps' sums of a strip meet in shared memory; a strip that a cut divides is finished by the last of its CTAs to
// arrive, which adds the parts in the order of the CTAs.  So all sums are taken in one fixed order.
// (Cutting at strips instead left 256 strips of 16 rows to 148 CTAs: 1.73 on average, 2 on the busiest.)
//
// Columns.  Products with 16-bit weights take the weights' type.  An input that has more bits than one column holds is split
// over several: bf16 products take f16 in two and f32 in three columns; binary16 products take a token times the power of
// two that brings its largest magnitude to [2^13, 2^14), in one column for bf16 and two for f32.  4-bit gate and up rows are
// multiplied as integers, with the token in fixed point as four columns of bytes (pp_q4.cu says how and why).  act is f32
// and always takes three columns: in bf16 these are its 24 bits; in binary16 (4-bit experts too) they hold v * 2^-11, the
// rest * 2^-1 and the rest * 2^10, which together are v to 24 bits between 2^-11 and 2^27 and to an absolute 2^-35 below.  No
// element's size is known before all of act is, but a bound is: |G x| |U x| <= |G| |U| |x|^2 in norms of rows and token.  v is
// act times the token's power of two that brings this bound to 2^26, so it cannot overflow, and 24 bits hold down to 2^-35 of
// the bound (powers of two are up to 4 above it); with random rows the bound is about H times a typical element.  y takes the power of two back.
//
// us in a graph and called one after another: 64 experts of 4096 x 2048, 8 a token, bf16, 16 tokens 453 (6.3 TB/s) and 487; 64 of
// 2048 x 1024, 4 tokens, 4 bits 33.0 and 35.5 (of 13 for the bytes: bound by instructions); 8 experts of 1024, 2 a token, one
// token 13.2 and 14.3 (bound by the steps' latency).
#include "pp_q4.cuh"

#include <algorithm>
#include <cmath>
#include <new>

namespace pp {
extern int g_stream_wait_polls;
}

struct pp_moe {
    int E, H, F, top_k, renorm, max_tokens, wtype, sets;      // wtype: PP_F16, PP_BF16 or -1 for 4-bit codes
    bool asym, bf16_scales;
    int act_bound;
    int strips1, strips2, kb1, kb2;
    int device, ctas;         // ctas: that the device holds at once
    unsigned char *gate_up, *down, *gate_up_sets, *down_sets;
    float *router, *logits, *xscale;
    uint16_t *xcols, *acols;
    int* xmeta;
    float* parts;             // [CTA][2][16][width]: its parts of the strips that its first and last cut divide
    int* sync;                // [0], [1] arrivals at the two barriers, [2] CTAs that are done, [3] status, then arrivals at
                              // divided strips, [step][the first of the strip's CTAs]
};

namespace pp {
namespace {

constexpr int kWarps = 16, kThreads = kWarps * 32, kMaxCols = 16;
constexpr int kMaxExperts = 256, kMaxTopK = 16, kMaxTokens = 32, kActCols = 3, kMaxCap = kMaxCols / kActCols;
constexpr int kByteCols = byte_columns<float>();      // of a token with 4-bit experts
constexpr int kRouterParts = 2;            // of a logit, at most
constexpr int kSpinPolls = 1 << 24;          // seconds; a barrier that is met never gets near it

struct MoeArgs {
    const unsigned char *gate_up, *down, *gate_up_sets, *down_sets;       // units, and their sets of 4-bit scales
    const float* router;
    XIn in;
    float *logits, *xscale, *parts;           // xscale: [tokens] of the inputs, then [tokens] of act
    uint16_t *xcols, *acols;
    int* xmeta;                              // 4-bit experts: [token's column][block] {its sums over the sets, its scale}
    int* sync;
    void* y;
    int32_t* ids;
    float* gates;
    int y_type, T, E, H, top_k, renorm, strips1, strips2, kb1, kb2, kpad1, kpad2, router_ld, slot_bytes, cpt, bf16_scales, polls;
    int router_parts, router_cols;           // parts of a logit, columns of a part
    float per_expert, per_entry, per_kb1, per_cta, per_cap, per_top_k;       // 1 / strips1, 1 / kb2, 1 / kb1, 1 / grid, ...
    double per_cta64;
    int round_log2;                          // of the strips of a round
    int round;                               // strips of a round
    int cap;                                 // tokens of an entry, at most
    int list_off, scr_off, park_off;         // shared memory; the weight rings are at 0
    int act_bound;                           // |row of G| |row of U| <= 2^act_bound
    int bytes_off;                           // 4-bit experts: where the tokens' bytes go, 0 if they stay in global memory
};

// ---- weight formats: bytes and columns of a unit, and its product with the columns a lane reads ------------------
__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint4& a, uint32_t b0, uint32_t b1) {
    asm(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b0), "r"(b1));
}

// Cols<STEP>: what a lane holds of one tile of 8 columns for a unit.
template <bool BF16> struct Wide {           // 16-bit weights: 16 rows x 32 columns, two operand fragments of 512 bytes
    static constexpr int kUnitCols = 32, kSetBytes = 0;
    static constexpr bool kBf16 = BF16, kBytes = false, kSwap = false;
    template <int STEP> struct Cols { uint4 x[1]; };
    template <int STEP, int NT>
    static __device__ __forceinline__ void unit(float (&tot)[NT][4], const unsigned char* slot, int lane, bool, const Cols<STEP>* x) {
        const uint4 a = at<uint4>(slot + lane * 16), b = at<uint4>(slot + 512 + lane * 16);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const uint4 v = x[nt].x[0];
            // the instruction cuts what its sum cannot hold; over a long row the cuts would add up, all towards zero, so
            // each unit's sum is rounded into the total
            float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            if (BF16) {
                mma_bf16(acc, a, v.x, v.y);
                mma_bf16(acc, b, v.z, v.w);
            } else {
                const uint32_t ar[4] = {a.x, a.y, a.z, a.w}, br[4] = {b.x, b.y, b.z, b.w};
                mma_f16(acc, ar, v.x, v.y);
                mma_f16(acc, br, v.z, v.w);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) tot[nt][i] += acc[i];
        }
    }
};

template <int SETS, bool ASYM> struct Q4 {
    static constexpr int kUnitCols = kQ4UnitCols, kSetBytes = SETS * (ASYM ? 48 : 32), kMeta = SETS == 1 ? 2 : SETS == 2 ? 4 : 8;
    static constexpr int kSets = SETS;
    static constexpr bool kBf16 = false, kBytes = true;       // kBytes: step 1 multiplies whole numbers
    static constexpr bool kSwap = true;                       // columns 4i + 1 and 4i + 2 of act change places
    template <int STEP> struct Cols {                         // step 1: 16 bytes of each 64 columns; sums and scales of two result columns
        uint4 x[STEP == 1 ? 2 : 4];
        alignas(16) int meta[2][STEP == 1 ? kMeta : 4];
    };
    template <int STEP, int NT>
    static __device__ __forceinline__ void unit(float (&tot)[NT][4], const unsigned char* slot, int lane, bool bf16_scales, const Cols<STEP>* x) {
        if constexpr (STEP == 1) {
            q4_unit_i8<NT, SETS, ASYM>(tot, slot, lane, bf16_scales, [&](int nt, int h) { return x[nt].x[h]; },
                                       [&](int nt, int set) { return make_int2(x[nt].meta[0][set], x[nt].meta[1][set]); },
                                       [&](int nt) { return make_float2(__int_as_float(x[nt].meta[0][SETS]), __int_as_float(x[nt].meta[1][SETS])); });
        } else {
            q4_unit_f16<NT, SETS, ASYM>(tot, slot, lane, bf16_scales, [&](int nt, int j) { return x[nt].x[j]; },
                                        [](int) { return make_float2(1.0f, 1.0f); });
        }
    }
};

// The columns of 16-bit experts' units (512 bytes a tile) travel in the ring with the weights: read through L1 instead, the
// first pass of a CTA over a new expert's columns took twice as long as the others, a trip to L2 per unit.  4-bit experts
// read the tokens' bytes in step 1 from shared memory, where they are few enough, and act in step 2 through L1, a unit
// ahead (2 KB a tile beside 1 KB of weights: in a ring of three units, all that fit, step 2 took 5 % longer).
__host__ __device__ constexpr int pad128(int n) { return (n + 127) / 128 * 128; }       // slots and their parts start on 128 bytes
// Units in flight per warp.
template <class W, int TILES> __host__ __device__ constexpr int depth() { return !W::kBytes && TILES == 2 ? 4 : 6; }

// ---- small helpers -----------------------------------------------------------------------------------------------
// Grid barrier in two parts.  After the second every CTA of the grid has passed the first and what it wrote before is
// visible; false if the wait gave up.
__device__ __forceinline__ void grid_arrive(int* counter) {
    __syncthreads();
    if (threadIdx.x == 0) asm volatile("red.release.gpu.global.add.s32 [%0], 1;" ::"l"(counter) : "memory");
}
__device__ __forceinline__ bool grid_wait(const int* counter, int* status, int polls, int* flag) {
    if (threadIdx.x == 0) {
        const int limit = polls > 0 ? polls : kSpinPolls;
        int seen = 0;
        for (int i = 0; i < limit; ++i) {
            asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(seen) : "l"(counter) : "memory");
            if (seen >= (int)gridDim.x) break;
        }
        *flag = seen >= (int)gridDim.x;
        if (!*flag) *status = 1;
    }
    __syncthreads();
    return *flag != 0;
}

__device__ __forceinline__ void warm(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }

__device__ __forceinline__ void store_y(void* y, int64_t i, int type, float v) {
    if (type == PP_F32) static_cast<float*>(y)[i] = v;
    else if (type == PP_F16) static_cast<__half*>(y)[i] = __float2half_rn(v);
    else static_cast<__nv_bfloat16*>(y)[i] = __float2bfloat16_rn(v);
}

template <bool BF16> __device__ __forceinline__ float round16(float v, uint16_t& bits) {
    if (BF16) {
        const __nv_bfloat16 h = __float2bfloat16_rn(v);
        bits = __bfloat16_as_ushort(h);
        return __bfloat162float(h);
    }
    const __half h = __float2half_rn(v);
    bits = __half_as_ushort(h);
    return __half2float(h);
}

// The columns of one value (see above), `step` elements apart.
template <bool BF16> __device__ __forceinline__ void split_act(float v, uint16_t* dst, int64_t step) {
    uint16_t b;
    if (BF16) {
        for (int c = 0; c < kActCols; ++c) {
            v -= round16<true>(v, b);
            dst[c * step] = b;
        }
    } else {
        v -= round16<false>(v * 0x1p-11f, b) * 0x1p11f;
        dst[0] = b;
        v -= round16<false>(v * 0x1p-1f, b) * 2.0f;
        dst[step] = b;
        round16<false>(v * 0x1p10f, b);
        dst[2 * step] = b;
    }
}

// The power of two of a token's act: 2^26 / (a bound of its elements), sum: the squares of the token.  Every fp32 number times
// the smallest, 2^-101, still fits the three columns.
__device__ __forceinline__ float act_scale(float sum, int act_bound) {
    const int e = (int)(__float_as_uint(sum) >> 23 & 255u) - 126;         // sum < 2^e
    return __uint_as_float((uint32_t)(min(max(26 - e - act_bound, -101), 126) + 127) << 23);
}
__device__ __forceinline__ float inverse_power(float p) { return __uint_as_float((254u << 23) - __float_as_uint(p)); }

// Columns a token takes.
template <bool BF16, typename T> __host__ __device__ constexpr int columns() {
    return std::is_same_v<T, float> ? (BF16 ? 3 : 2) : BF16 && std::is_same_v<T, __half> ? 2 : 1;
}

// ---- step 0 ------------------------------------------------------------------------------------------------------
// One CTA turns a token into columns.
template <class W, typename T, bool VEC> __device__ __forceinline__ void token_columns(const MoeArgs& a, int token, float* part) {
    constexpr bool BF16 = W::kBf16;
    constexpr int cpt = columns<BF16, T>();
    const T* x = static_cast<const T*>(a.in.x) + (int64_t)token * a.in.ld;
    float up = 1.0f, down = 1.0f, act = 1.0f;
    if (!BF16) {
        float most = 0.0f, sum = 0.0f;
#pragma unroll 2
        for (int c = threadIdx.x * 4; c < a.H; c += kThreads * 4) {
            const Pack<T, 4> v = load_four<VEC>(x, c, a.H);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float f = to_float(v.v[i]);
                most = fmaxf(most, fabsf(f));
                sum = fmaf(f, f, sum);
            }
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
            sum += __shfl_xor_sync(0xffffffffu, sum, o);
        }
        __syncthreads();                                     // an earlier token's values have been read
        if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = most, part[kWarps + (threadIdx.x >> 5)] = sum;
        __syncthreads();
        most = part[threadIdx.x & (kWarps - 1)];
        sum = part[kWarps + (threadIdx.x & (kWarps - 1))];
#pragma unroll
        for (int o = kWarps / 2; o; o >>= 1) {
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
            sum += __shfl_xor_sync(0xffffffffu, sum, o);
        }
        if (!std::is_same_v<T, __half>) f16_scale(most, up, down);
        act = act_scale(sum, a.act_bound);
    }
    uint16_t* dst = a.xcols + (int64_t)token * cpt * a.kpad1;
#pragma unroll 2
    for (int c = threadIdx.x * 4; c < a.kpad1; c += kThreads * 4) {       // zeros up to the padded length
        const Pack<T, 4> v = load_four<VEC>(x, c, a.H);
        Pack<uint16_t, 4> bits[cpt];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float rest = to_float(v.v[i]) * up;
#pragma unroll
            for (int k = 0; k < cpt; ++k) rest -= round16<BF16>(rest, bits[k].v[i]);
        }
#pragma unroll
        for (int k = 0; k < cpt; ++k) *reinterpret_cast<Pack<uint16_t, 4>*>(dst + (int64_t)k * a.kpad1 + c) = bits[k];
    }
    if (threadIdx.x == 0) a.xscale[token] = down, a.xscale[a.T + token] = act;
}

// The same for 4-bit experts: a warp per block of 128 columns.
template <int SETS, int META, typename T, bool VEC> __device__ __forceinline__ void token_bytes(const MoeArgs& a, int token, float* part) {
    const int lane = threadIdx.x & 31;
    float squares = 0.0f;
    const T* x = static_cast<const T*>(a.in.x) + (int64_t)token * a.in.ld;
    for (int kb = threadIdx.x >> 5; kb < a.kb1; kb += kWarps) {
        uint32_t w[kByteCols];
        float down;
        const Pack<T, 4> v = load_four<VEC>(x, kb * kQ4UnitCols + lane * 4, a.H);
        fixed_point(v, 1.0f, w, down);
#pragma unroll
        for (int i = 0; i < 4; ++i) squares = fmaf(to_float(v.v[i]), to_float(v.v[i]), squares);
        unsigned char* dst = reinterpret_cast<unsigned char*>(a.xcols) + (int64_t)token * kByteCols * a.kpad1 + kb * kQ4UnitCols + byte_offset(lane);
#pragma unroll
        for (int c = 0; c < kByteCols; ++c) *reinterpret_cast<uint32_t*>(dst + (int64_t)c * a.kpad1) = w[c];
        const int sum = byte_sums<SETS>(w, lane), c = lane & (32 / SETS - 1);
        if (c < kByteCols) {
            int* meta = a.xmeta + ((int64_t)(token * kByteCols + c) * a.kb1 + kb) * META;
            meta[lane / (32 / SETS)] = sum;
            if (lane < kByteCols) meta[SETS] = __float_as_int(down * byte_weight<kByteCols>(c));
        }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) squares += __shfl_xor_sync(0xffffffffu, squares, o);
    __syncthreads();                                         // an earlier token's have been read
    if (lane == 0) part[threadIdx.x >> 5] = squares;
    __syncthreads();
    if (threadIdx.x == 0) {
        squares = 0.0f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) squares += part[w];
        a.xscale[token] = 1.0f;
        a.xscale[a.T + token] = act_scale(squares, a.act_bound);
    }
}

// A warp's part of the logit of one (token, expert): columns from .. to.
template <typename T, bool VEC> __device__ __forceinline__ float router_part(const MoeArgs& a, int token, int expert, int from, int to) {
    constexpr int kAhead = VEC ? 4 : 1;
    const int lane = threadIdx.x & 31;
    const float* r = a.router + (int64_t)expert * a.router_ld;
    const T* row = static_cast<const T*>(a.in.x) + (int64_t)token * a.in.ld;
    float sum = 0.0f;
#pragma unroll 1
    for (int c0 = from + lane * 4; c0 < to; c0 += kAhead * 128) {
        Pack<T, 4> x[kAhead];
        float4 w[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            x[i] = load_four<VEC>(row, c0 + i * 128, to);                  // zeros past the end: the router's row may repeat there
            w[i] = __ldg(reinterpret_cast<const float4*>(r + min(c0 + i * 128, a.router_ld - 4)));
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            sum = fmaf(to_float(x[i].v[0]), w[i].x, sum);
            sum = fmaf(to_float(x[i].v[1]), w[i].y, sum);
            sum = fmaf(to_float(x[i].v[2]), w[i].z, sum);
            sum = fmaf(to_float(x[i].v[3]), w[i].w, sum);
        }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    return sum;
}

// Parts of logits go to warp 0 of every CTA, the last CTA first (the first ones have tokens to turn into columns), then to
// warp 1 and so on; a row is cut into as many parts as keep every warp at one.
template <class W, typename T, bool VEC> __device__ __forceinline__ void step0(const MoeArgs& a, float* part) {
    for (int t = blockIdx.x; t < a.T; t += gridDim.x) {
        if constexpr (W::kBytes) token_bytes<W::kSets, W::kMeta, T, VEC>(a, t, part);
        else token_columns<W, T, VEC>(a, t, part);
    }
    for (int i = (threadIdx.x >> 5) * gridDim.x + (gridDim.x - 1 - blockIdx.x); i < a.T * a.E * a.router_parts; i += kWarps * gridDim.x) {
        const int k = i / (a.T * a.E), pair = i - k * a.T * a.E, from = k * a.router_cols;
        const float v = router_part<T, VEC>(a, pair / a.E, pair % a.E, from, min(a.H, from + a.router_cols));
        if ((threadIdx.x & 31) == 0) a.logits[i] = v;
    }
}
template <class W, typename T> __device__ __forceinline__ void step0(const MoeArgs& a, float* part) {
    if (a.in.vec) step0<W, T, true>(a, part);
    else step0<W, T, false>(a, part);
}

// x / n from the reciprocal of n, for quotients below 2^21.
__device__ __forceinline__ int divide(int x, int n, float r) {
    int q = (int)((float)x * r);
    const int rest = x - q * n;
    if (rest < 0) --q;
    if (rest >= n) ++q;
    return q;
}

// ---- routing, by every CTA for itself ----------------------------------------------------------------------------
struct Lists {
    int4* entry;         // {expert, first pair, pairs, 0}: an expert and up to `cap` of its tokens
    int2* plan;          // [32, the most strips of a round] {which warps have sums of it, its entry (step 1)}
    int* pair_token;     // pairs (token, expert) in the order of the experts
    float* pair_gate;
    int* chosen;         // [T][top_k] experts
    float* gate;         // [T][top_k]
    float* xscale;       // [T], then act's [T]
    uint32_t* tokens;    // [E] which tokens chose the expert
    int* first;          // [E] its first pair
    int* sums;           // [warps] scratch of the scan
    const unsigned char* xbytes;     // 4-bit experts: the tokens' bytes and what is kept of them, in shared memory where they fit
    const int* xmeta;
    int* cuts;           // [2][2] first and last CTA of the strips that the CTA's ends divide, [4..5] whether it finishes them
};
__host__ __device__ inline int list_bytes(int T, int E, int top_k) {
    return (T * top_k * (16 + 4 + 4 + 4 + 4) + 32 * 8 + T * 8 + E * 8 + 16 * 4 + 8 * 4 + 127) / 128 * 128;
}
__device__ __forceinline__ Lists lists_at(unsigned char* p, int T, int E, int top_k) {
    Lists L;
    const int n = T * top_k;
    L.entry = reinterpret_cast<int4*>(p);
    L.plan = reinterpret_cast<int2*>(L.entry + n);
    L.pair_token = reinterpret_cast<int*>(L.plan + 32);
    L.pair_gate = reinterpret_cast<float*>(L.pair_token + n);
    L.chosen = reinterpret_cast<int*>(L.pair_gate + n);
    L.gate = reinterpret_cast<float*>(L.chosen + n);
    L.xscale = L.gate + n;
    L.tokens = reinterpret_cast<uint32_t*>(L.xscale + 2 * T);
    L.first = reinterpret_cast<int*>(L.tokens + E);
    L.sums = L.first + E;
    L.cuts = L.sums + 16;
    return L;
}

// A warp chooses a token's experts: the largest logit's key (floats as whole numbers in the same order) top_k times, among
// equal ones the lowest index; lane j keeps the j-th.  Then the softmax over them, or over all.
template <int kEach> __device__ __forceinline__ void choose(const MoeArgs& a, const Lists& L, int t) {       // kEach: logits of a lane
    const int lane = threadIdx.x & 31;
    const float* row = a.logits + t * a.E;                   // [part][token][expert]
    uint32_t key[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        key[i] = 0u;                                         // below every logit
        if (i * 32 + lane < a.E) {
            float v[kRouterParts], l = 0.0f;
#pragma unroll
            for (int k = 0; k < kRouterParts; ++k) v[k] = k < a.router_parts ? __ldcg(row + k * a.T * a.E + i * 32 + lane) : 0.0f;
#pragma unroll
            for (int k = 0; k < kRouterParts; ++k) l += v[k];
            const uint32_t u = __float_as_uint(l == l ? l : -INFINITY);    // what cannot be compared ranks last
            key[i] = (int)u < 0 ? ~u : u | 0x80000000u;
        }
    }
    uint32_t mine = 0u;
    int expert = 0;
    for (int j = 0; j < a.top_k; ++j) {
        uint32_t most = key[0];
#pragma unroll
        for (int i = 1; i < kEach; ++i) most = max(most, key[i]);
        most = __reduce_max_sync(0xffffffffu, most);
        uint32_t at = 0xffffffffu;
#pragma unroll
        for (int i = kEach - 1; i >= 0; --i)
            if (key[i] == most) at = i * 32 + lane;
        at = __reduce_min_sync(0xffffffffu, at);
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (at == i * 32 + lane) key[i] = 0u;
        if (lane == j) mine = most, expert = (int)at;
    }
    const uint32_t u = (int)mine < 0 ? mine & 0x7fffffffu : ~mine;
    const float l = __uint_as_float(u), most0 = __shfl_sync(0xffffffffu, l, 0);
    float p = lane < a.top_k ? expf(l - most0) : 0.0f, sum = p;
    if (!a.renorm) {                                         // the experts that were not chosen count as well
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (key[i]) {
                const uint32_t v = (int)key[i] < 0 ? key[i] & 0x7fffffffu : ~key[i];
                sum += expf(__uint_as_float(v) - most0);
            }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    p /= sum;
    int rank = 0;
    if (a.T == 1)
        for (int j = 0; j < a.top_k; ++j) rank += __shfl_sync(0xffffffffu, expert, j) < expert;
    if (lane < a.top_k) {
        const int at = t * a.top_k + lane;
        if (a.T == 1) {                                      // every expert has one pair: its place is its rank
            L.entry[rank] = make_int4(expert, rank, 1, 0);
            L.pair_token[rank] = 0;
            L.pair_gate[rank] = p;
        } else {
            L.chosen[at] = expert;
            L.gate[at] = p;
            atomicOr(L.tokens + expert, 1u << t);
        }
        if (blockIdx.x == 0) {
            if (a.ids) a.ids[at] = expert;
            if (a.gates) a.gates[at] = p;
        }
    }
}

__device__ __forceinline__ int route(const MoeArgs& a, const Lists& L) {       // the number of entries; L.tokens is zero before
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const float xscale = tid < 2 * a.T ? __ldcg(a.xscale + tid) : 0.0f;       // stored behind the choice, which would wait for it
    for (int t = warp; t < a.T; t += kWarps) {
        if (a.E <= 32) choose<1>(a, L, t);
        else if (a.E <= 64) choose<2>(a, L, t);
        else choose<kMaxExperts / 32>(a, L, t);
    }
    if (tid < 2 * a.T) L.xscale[tid] = xscale;
    __syncthreads();
    if (a.T == 1) return a.top_k;                            // its lists are made (8 experts: 13.3 us, through the counts below 13.6)
    // where each expert's pairs and entries start: both counts in one scan (neither exceeds 512)
    const int n = tid < a.E ? __popc(L.tokens[tid]) : 0;
    const int mine = n | divide(n + a.cap - 1, a.cap, a.per_cap) << 16;
    int both = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, both, o);
        if (lane >= o) both += v;
    }
    if (lane == 31) L.sums[warp] = both;
    __syncthreads();
    int before = both - mine, all = 0;
#pragma unroll
    for (int w = 0; w < kMaxExperts / 32; ++w) {
        const int v = L.sums[w];
        if (w < warp) before += v;
        all += v;
    }
    if (n) {
        const int first = before & 0xffff, entry = before >> 16;
        L.first[tid] = first;
        for (int i = 0; i * a.cap < n; ++i) L.entry[entry + i] = make_int4(tid, first + i * a.cap, min(a.cap, n - i * a.cap), 0);
    }
    __syncthreads();
    if (tid < a.T * a.top_k) {                               // at most 512 pairs
        const int t = divide(tid, a.top_k, a.per_top_k), e = L.chosen[tid], p = L.first[e] + __popc(L.tokens[e] & ((1u << t) - 1u));
        L.pair_token[p] = t;
        L.pair_gate[p] = L.gate[tid];
    }
    __syncthreads();
    return all >> 16;
}

// ---- steps 1 and 2: the stream of weights ------------------------------------------------------------------------
// Units are numbered strip after strip, nv to a strip: in step 1 the blocks of the columns of x (a strip belongs to one
// entry), in step 2 the entries' blocks of the columns of act, one entry after another (a strip is 16 rows of y).  A CTA
// has units begin .. end; x below counts them from the start of its first strip, x0 .. x1, and a round is `round` strips.
struct Span {
    int nv, ctas, first, x0, x1, rounds, strips;     // ctas: that have units at all; first: the first strip; strips: of this CTA
    float per_strip;                                 // 1 / nv
    bool whole;                                      // no strip is divided
};
struct Run { const unsigned char *unit, *sets; int left, ls, entry, kb; };        // units that lie one after another; ls: strip - first

// This CTA's part of `strips` strips of nv units.  Cuts fall between strips unless that leaves the busiest CTA with kJoin
// units more than its equal share: joining a divided strip takes about 3,700 cycles, 84 units at the rate of HBM (148 CTAs:
// 256 strips of 32 units are faster whole, 256 strips of 3,600 units are not: 519,000 cycles whole, 396,000 cut).
constexpr int kJoin = 84;
// (Divisions by reciprocals: a CTA's way from the choice to its first copies holds four of them.)
__device__ __forceinline__ Span span_of(const MoeArgs& a, int strips, int nv, float per_strip) {
    Span s;
    s.nv = nv;
    s.per_strip = per_strip;
    const int grid = (int)gridDim.x, cta = (int)blockIdx.x;
    const int each = divide(strips, grid, a.per_cta), more = strips - each * grid;   // strips of a CTA, CTAs with one more
    s.whole = (int64_t)(more ? grid - more : 0) * nv <= (int64_t)kJoin * grid;
    if (s.whole) {
        s.ctas = min(grid, strips);
        s.first = each * cta + min(cta, more);
        s.x0 = 0;
        s.strips = each + (cta < more);
        s.x1 = s.strips * nv;
    } else {
        const int64_t units = (int64_t)strips * nv;           // below 2^34
        s.ctas = (int)min((int64_t)grid, units);
        const auto start = [&](int c) {                       // units * c / ctas
            if (units <= grid) return min((int64_t)c, units);
            const int64_t n = units * c;                      // below 2^53
            int64_t q = (int64_t)((double)n * a.per_cta64);
            const int64_t rest = n - q * grid;
            return rest < 0 ? q - 1 : rest >= grid ? q + 1 : q;
        };
        const int64_t begin = start(cta), end = start(cta + 1);
        int first = (int)((float)begin * per_strip);          // at most 2^22 strips: off by one at most
        const int64_t rest = begin - (int64_t)first * nv;
        s.first = first += rest < 0 ? -1 : rest >= nv ? 1 : 0;
        s.x0 = (int)(begin - (int64_t)first * nv);
        s.x1 = s.x0 + (int)(end - begin);
        s.strips = s.x1 > s.x0 ? divide(s.x1 + nv - 1, nv, per_strip) : 0;
    }
    s.rounds = (s.strips + a.round - 1) >> a.round_log2;
    return s;
}

template <class W, int STEP> __device__ __forceinline__ void locate(const MoeArgs& a, const Lists& L, const Span& s, int x, int stop, Run& r) {
    r.ls = divide(x, s.nv, s.per_strip);
    const int v = x - r.ls * s.nv;
    int strip = s.first + r.ls;
    if (STEP == 1) {
        r.entry = divide(strip, a.strips1, a.per_expert);
        strip -= r.entry * a.strips1;
        r.kb = v;
        r.left = min(s.nv - v, stop - x);
    } else {
        r.entry = divide(v, a.kb2, a.per_entry);
        r.kb = v - r.entry * a.kb2;
        r.left = min(a.kb2 - r.kb, stop - x);
    }
    const int64_t at = ((int64_t)L.entry[r.entry].x * (STEP == 1 ? a.strips1 : a.strips2) + strip) * (STEP == 1 ? a.kb1 : a.kb2) + r.kb;
    r.unit = (STEP == 1 ? a.gate_up : a.down) + at * 1024;
    r.sets = (STEP == 1 ? a.gate_up_sets : a.down_sets) + at * W::kSetBytes;
}

// This warp's units of a round: x .. stop (a round has at most 2^25 units).
__device__ __forceinline__ void warp_range(const Span& s, int round, int strips, int warp, int& x, int& stop) {
    const int lo = max(s.x0, round * strips * s.nv), n = min(s.x1, (round + 1) * strips * s.nv) - lo;
    x = lo + (int)((uint32_t)(n * warp) / kWarps);
    stop = lo + (int)((uint32_t)(n * (warp + 1)) / kWarps);
}

// Where a lane reads the columns of a run, from its first unit on: its input column 8 nt + g of the entry's tiles and, of
// bytes, what is kept of its two result columns.
template <class W, int STEP, int TILES> struct ColumnsAt {
    static constexpr bool kBytes = W::kBytes && STEP == 1;
    const unsigned char* x[TILES];
    const int* meta[kBytes ? TILES : 1][2];
    __device__ __forceinline__ void set(const MoeArgs& a, const Lists& L, const Run& r, int lane, int tiles) {
        const int cpt = STEP == 1 ? a.cpt : kActCols;
        const int4 entry = L.entry[r.entry];
        const auto row = [&](int c) {                        // columns past the last repeat one
            const int pl = kBytes ? c / kByteCols : cpt == 1 ? c : cpt == 2 ? c >> 1 : c / 3, p = entry.y + min(pl, entry.z - 1);
            return (STEP == 1 ? L.pair_token[p] : p) * cpt + c - pl * cpt;
        };
#pragma unroll
        for (int nt = 0; nt < TILES; ++nt) {
            if (nt >= tiles) break;
            const int64_t at = (int64_t)row(nt * 8 + (lane >> 2)) * (STEP == 1 ? a.kpad1 : a.kpad2) + r.kb * W::kUnitCols;
            x[nt] = (kBytes ? L.xbytes : reinterpret_cast<const unsigned char*>(STEP == 1 ? a.xcols : a.acols) + at) + at + (lane & 3) * 16;
            if constexpr (kBytes) {
#pragma unroll
                for (int i = 0; i < 2; ++i) meta[nt][i] = L.xmeta + (row(nt * 8 + (lane & 3) * 2 + i) * a.kb1 + r.kb) * W::kMeta;
            }
        }
    }
    __device__ __forceinline__ void advance() {
#pragma unroll
        for (int nt = 0; nt < TILES; ++nt) {
            x[nt] += W::kUnitCols * (kBytes ? 1 : 2);
            if constexpr (kBytes) meta[nt][0] += W::kMeta, meta[nt][1] += W::kMeta;
        }
    }
    __device__ __forceinline__ void read(typename W::template Cols<STEP> (&c)[TILES], int tiles) const {
#pragma unroll
        for (int nt = 0; nt < TILES; ++nt) {
            if (nt >= tiles) break;
#pragma unroll
            for (int j = 0; j < (int)(sizeof(c[nt].x) / 16); ++j) c[nt].x[j] = *reinterpret_cast<const uint4*>(x[nt] + j * 64);
            if constexpr (kBytes) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if constexpr (W::kMeta == 2) {
                        *reinterpret_cast<int2*>(c[nt].meta[i]) = *reinterpret_cast<const int2*>(meta[nt][i]);
                    } else {
#pragma unroll
                        for (int k = 0; k < W::kMeta; k += 4) *reinterpret_cast<int4*>(c[nt].meta[i] + k) = *reinterpret_cast<const int4*>(meta[nt][i] + k);
                    }
                }
            }
        }
    }
};

// A warp's asynchronous copies, unit after unit of its runs.
template <class W, int STEP, int TILES> struct Fetcher {
    int round = -1, x = 0, stop = 0, left = 0, tiles = 1;    // x: where the next run starts, left: units of this one
    const unsigned char *unit = nullptr, *sets = nullptr;    // this lane's bytes of them
    ColumnsAt<W, STEP, TILES> from;
    __device__ __forceinline__ void next(const MoeArgs& a, const Lists& L, const Span& s, int warp, int lane, uint32_t slot, bool weights, bool cols) {
        if (left == 0) {
            while (x == stop && round < s.rounds)
                if (++round < s.rounds) warp_range(s, round, a.round, warp, x, stop);
            if (x < stop) {
                Run r;
                locate<W, STEP>(a, L, s, x, stop, r);
                x += left = r.left;
                unit = r.unit + lane * 16;
                sets = r.sets + lane * 16;
                if (TILES > 1) tiles = (L.entry[r.entry].z * (STEP == 1 ? a.cpt : kActCols) + 7) / 8;
                if (!W::kBytes) from.set(a, L, r, lane, tiles);
            }
        }
        if (left) {
            --left;
            if (weights) {
                cp_async16(slot, unit);
                cp_async16(slot + 512, unit + 512);
                if (lane < W::kSetBytes / 16) cp_async16(slot + 1024, sets);
            }
            unit += 1024;
            sets += W::kSetBytes;
            if (!W::kBytes) {
#pragma unroll
                for (int nt = 0; nt < TILES; ++nt)
                    if (cols && nt < tiles) cp_async16_l1(slot + 1024 + nt * 512, from.x[nt]);
                from.advance();
            }
        }
        cp_commit();
    }
};

// What a strip's sums become.  Step 1: act of one (row, pair), step 2: y of one (row, token).
template <class W> __device__ __forceinline__ void finish_act(const MoeArgs& a, const Lists& L, int entry, int strip, int row8, int pl, float gate, float up) {
    const int p = L.entry[entry].y + pl, row = (strip - entry * a.strips1) * 8 + row8;
    const int token = L.pair_token[p];
    const float scale = L.xscale[token];
    gate *= scale;
    up *= scale;
    float act = L.pair_gate[p] * (__fdividef(gate, 1.0f + expf(-gate)) * up);
    if (!W::kBf16) act *= L.xscale[a.T + token];
    const int at = W::kSwap && ((row & 3) == 1 || (row & 3) == 2) ? row ^ 3 : row;
    split_act<W::kBf16>(act, a.acols + (int64_t)p * kActCols * a.kpad2 + at, a.kpad2);
}
template <class W> __device__ __forceinline__ void finish_y(const MoeArgs& a, const Lists& L, int strip, int row, int token, float v) {
    const int m = strip * 16 + row;
    if (!W::kBf16) v *= inverse_power(L.xscale[a.T + token]);
    if (m < a.H) store_y(a.y, (int64_t)token * a.H + m, a.y_type, v);
}

template <class W, int STEP, int TILES>
__device__ __forceinline__ void stream(const MoeArgs& a, const Lists& L, const Span& s, Fetcher<W, STEP, TILES>& f, unsigned char* smem) {
    constexpr int kDepth = depth<W, TILES>(), kCols = 8 * TILES;
    constexpr bool kRing = !W::kBytes;                       // columns come with the weights
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int cpt = STEP == 1 ? a.cpt : kActCols, width = STEP == 1 ? a.cap : a.T;
    unsigned char *ring = smem + warp * kDepth * a.slot_bytes, *ring_end = ring + kDepth * a.slot_bytes, *at = ring;
    float* scr = reinterpret_cast<float*>(smem + a.scr_off) + warp * 16 * kCols;
    float* park = reinterpret_cast<float*>(smem + a.park_off);
    float* my_parts = a.parts + (int64_t)blockIdx.x * 2 * 16 * width;
    // the strips that the CTA's ends divide: its first and its last (one, if it has only one)
    const bool cut_first = s.strips && s.x0 > 0, cut_last = s.strips && s.x1 < s.strips * s.nv;
    for (int round = 0; round < s.rounds; ++round) {
        const int ls0 = round * a.round, rs = min(a.round, s.strips - ls0);
        int x, stop, strip = -1, tiles = 1;
        {                                                    // which warps will have sums of each strip: half a warp per strip
            const int q = tid >> 4, w = tid & 15;
            int lo, hi;
            warp_range(s, round, a.round, w, lo, hi);
            const bool has = q < rs && max(lo, (ls0 + q) * s.nv) < min(hi, (ls0 + q + 1) * s.nv);
            const uint32_t mask = __ballot_sync(0xffffffffu, has) >> (lane & 16) & 0xffffu;
            if (w == 0 && q < rs) L.plan[q] = make_int2((int)mask, STEP == 1 ? divide(s.first + ls0 + q, a.strips1, a.per_expert) : 0);
        }
        warp_range(s, round, a.round, warp, x, stop);
        Run run;
        run.left = 0;
        ColumnsAt<W, STEP, TILES> from;
        typename W::template Cols<STEP> xr[TILES];           // what the lane needs of the next unit's columns
        int4 entry = make_int4(0, 0, 0, 0);
        float tot[TILES][4] = {};
        const auto begin_run = [&] {
            locate<W, STEP>(a, L, s, x, stop, run);
            x += run.left;
            entry = L.entry[run.entry];
            tiles = TILES == 1 ? 1 : (entry.z * cpt + 7) / 8;
            if (!kRing) {
                from.set(a, L, run, lane, tiles);
                from.read(xr, tiles);
            }
        };
        if (x < stop) begin_run();
        while (run.left) {
            do {
                cp_wait<kDepth - 1>();
                if (W::kBytes) __syncwarp();                   // sets are read by other lanes than copied them; nothing else is
                if (kRing) {
#pragma unroll
                    for (int nt = 0; nt < TILES; ++nt)
                        if (nt < tiles) xr[nt].x[0] = *reinterpret_cast<const uint4*>(at + 1024 + nt * 512 + lane * 16);
                }
                if (TILES == 1 || tiles == 1) W::template unit<STEP, 1>(reinterpret_cast<float(&)[1][4]>(tot), at, lane, a.bf16_scales != 0, xr);
                else W::template unit<STEP, TILES>(tot, at, lane, a.bf16_scales != 0, xr);
                --run.left;
                if (!kRing && run.left) {                   // in flight while the other warps compute
                    from.advance();
                    from.read(xr, tiles);
                }
                if (W::kBytes) __syncwarp();
                f.next(a, L, s, warp, lane, smem_addr(at) + lane * 16, true, true);
                at += a.slot_bytes;
                if (at == ring_end) at = ring;
            } while (run.left);
            // add a token's columns and park the sums: piece (warp, strip) has slot warp + strip.  The next run's first columns
            // are requested in between.
#pragma unroll
            for (int nt = 0; nt < TILES; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    scr[(g + (i >> 1) * 8) * kCols + nt * 8 + 2 * t + (i & 1)] = tot[nt][i];
                    tot[nt][i] = 0.0f;
                }
            const int first = entry.y, pairs = entry.z, ls = run.ls;
            if (x < stop) begin_run();
            float* tile = park + (warp + ls - ls0) * 16 * width;
            if (STEP == 2 && ls != strip) {                    // a new strip's sums of this warp
                strip = ls;
                for (int i = lane; i < 16 * width; i += 32) tile[i] = 0.0f;
            }
            __syncwarp();
            const int row = lane & 15;
            for (int pl = lane >> 4; pl < pairs; pl += 2) {
                const float* c = scr + row * kCols + pl * cpt;
                if (STEP == 1) {
                    float v = c[0];
                    for (int k = 1; k < cpt; ++k) v += c[k];
                    tile[pl * 16 + row] = v;
                } else {
                    const float v = W::kBf16 ? c[0] + c[1] + c[2] : fmaf(c[0], 0x1p11f, fmaf(c[1], 2.0f, c[2] * 0x1p-10f));
                    tile[L.pair_token[first + pl] * 16 + row] += v;
                }
            }
            __syncwarp();
        }
        __syncthreads();

        // The pieces of a row in the order of the warps.  With fewer strips than warps a strip has many: then four lanes take
        // every fourth warp's and add theirs up (16 reads behind one another took 1,000 cycles).
        const bool four = rs < kWarps;
        const int shift = four ? 2 : 0, sub = four ? tid & 3 : 0;
        const auto pieces = [&](uint32_t mask, int q, int at) {
            float v = 0.0f;
            for (mask &= four ? 0x1111u << sub : 0xffffu; mask; mask &= mask - 1) v += park[(__ffs((int)mask) - 1 + q) * 16 * width + at];
            if (four) {
                v += __shfl_xor_sync(0xffffffffu, v, 1);
                v += __shfl_xor_sync(0xffffffffu, v, 2);
            }
            return v;
        };
        // a divided strip's slot among this CTA's parts: 0 where an earlier CTA has begun it
        const auto cut = [&](int ls) { return (ls == 0 && cut_first) || (ls == s.strips - 1 && cut_last); };
        const auto part = [&](int ls) { return my_parts + (ls == 0 && cut_first ? 0 : 16 * width); };
        if (STEP == 1) {
            for (int o = tid >> shift; o < rs * 8; o += kThreads >> shift) {               // four: a warp has the eight rows of one strip
                const int q = o >> 3, row = o & 7, ls = ls0 + q;
                const int2 plan = L.plan[q];
                const int pairs = L.entry[plan.y].z;
                for (int pl = 0; pl < pairs; ++pl) {
                    const float gate = pieces((uint32_t)plan.x, q, pl * 16 + row), up = pieces((uint32_t)plan.x, q, pl * 16 + row + 8);
                    if (four && sub != (pl & 3)) continue;
                    if (!cut(ls)) {
                        finish_act<W>(a, L, plan.y, s.first + ls, row, pl, gate, up);
                    } else {
                        __stcg(part(ls) + pl * 16 + row, gate);
                        __stcg(part(ls) + pl * 16 + row + 8, up);
                    }
                }
            }
        } else {
            const int per_strip = 16 * a.T, outs = rs * per_strip;
            const Divider by_strip(per_strip);
            for (int o = tid >> shift; o < outs; o += kThreads >> shift) {                 // four: outs is a multiple of the warp's eight
                const int q = by_strip.div(o), r = o - q * per_strip, ls = ls0 + q;
                const float v = pieces((uint32_t)L.plan[q].x, q, r);
                if (sub) continue;
                if (!cut(ls)) finish_y<W>(a, L, s.first + ls, r & 15, r >> 4, v);
                else __stcg(part(ls) + r, v);
            }
        }
        __syncthreads();
    }
}

// First and last CTA of the strips that this CTA's ends divide (-1: it divides none there): unit x belongs to the last CTA
// c with units * c / ctas <= x.  Two threads, while the weights are on their way.
__device__ __forceinline__ void find_cuts(const Lists& L, const Span& s, int64_t units) {
    const int which = threadIdx.x;
    if (which < 2) {
        const bool cut_first = s.strips && s.x0 > 0, cut_last = s.strips && s.x1 < s.strips * s.nv;
        const bool cut = which == 0 ? cut_first : cut_last && !(cut_first && s.strips == 1);
        const int64_t lo = (int64_t)(s.first + (which == 0 ? 0 : s.strips - 1)) * s.nv;
        L.cuts[which] = cut ? (int)(((lo + 1) * s.ctas - 1) / units) : -1;
        L.cuts[2 + which] = cut ? (int)(((lo + s.nv) * s.ctas - 1) / units) : -1;
    }
}

// Divided strips: the last of a strip's CTAs to arrive adds the parts in the order of the CTAs.
template <class W, int STEP> __device__ __forceinline__ void join(const MoeArgs& a, const Lists& L, const Span& s) {
    const int tid = threadIdx.x, width = STEP == 1 ? a.cap : a.T;
    if (tid < 2 && L.cuts[tid] >= 0) {                       // behind the barrier that ended the last round
        int* arrived = a.sync + 4 + (STEP - 1) * gridDim.x + L.cuts[tid];
        int before;
        asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], 1;" : "=r"(before) : "l"(arrived) : "memory");
        const bool last = before == L.cuts[2 + tid] - L.cuts[tid];
        if (last) *arrived = 0;
        L.cuts[4 + tid] = last;
    } else if (tid < 2) {
        L.cuts[4 + tid] = 0;
    }
    __syncthreads();
    const int per_strip = STEP == 1 ? 8 * a.cap : 16 * a.T;
    for (int o = tid; o < 2 * per_strip; o += kThreads) {
        const int which = o >= per_strip, r = o - which * per_strip;
        if (!L.cuts[4 + which]) continue;
        const int c0 = L.cuts[which], c1 = L.cuts[2 + which], strip = s.first + (which == 0 ? 0 : s.strips - 1);
        const int pl = r >> 3, row = r & 7, entry = STEP == 1 ? divide(strip, a.strips1, a.per_expert) : 0;
        if (STEP == 1 && pl >= L.entry[entry].z) continue;
        const int at = STEP == 1 ? pl * 16 + row : r;
        float v[2] = {0.0f, 0.0f};
#pragma unroll 4
        for (int c = c0; c <= c1; ++c) {
            const float* part = a.parts + ((int64_t)c * 2 + (c == c0 ? 1 : 0)) * 16 * width + at;
            v[0] += __ldcg(part);
            if (STEP == 1) v[1] += __ldcg(part + 8);
        }
        if (STEP == 1) finish_act<W>(a, L, entry, strip, row, pl, v[0], v[1]);
        else finish_y<W>(a, L, strip, r & 15, r >> 4, v[0]);
    }
}

template <class W, int TILES> __global__ void __launch_bounds__(kThreads, 1) moe_kernel(const MoeArgs a) {
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ float part[2 * kWarps];
    __shared__ int flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    Lists L = lists_at(smem + a.list_off, a.T, a.E, a.top_k);
    pdl_release();
    // before the wait: the router's rows on their way to L2, and the translations of what is touched first
    for (int i = blockIdx.x * kThreads + threadIdx.x; i < a.E * a.router_ld / 32; i += gridDim.x * kThreads) warm(a.router + i * 32);
    if (threadIdx.x == 0) {
        warm(a.in.x);
        warm(a.logits);
        warm(a.xcols);
        warm(a.acols);
        warm(a.y);
        warm(a.parts);
    }
    for (int e = threadIdx.x; e < a.E; e += kThreads) L.tokens[e] = 0u;
    pdl_wait();

    if (a.in.type == PP_BF16) step0<W, __nv_bfloat16>(a, part);
    else if (a.in.type == PP_F16) step0<W, __half>(a, part);
    else step0<W, float>(a, part);
    grid_arrive(a.sync);
    bool ok = grid_wait(a.sync, a.sync + 3, a.polls, &flag);
    if (ok) {
        if constexpr (W::kBytes) {                            // the tokens' bytes are on their way while the experts are chosen
            L.xbytes = reinterpret_cast<const unsigned char*>(a.xcols);
            L.xmeta = a.xmeta;
            if (a.bytes_off) {
                const int n = a.T * kByteCols * a.kpad1 / 16, m = (a.T * kByteCols * a.kb1 * W::kMeta + 3) / 4;
                for (int i = threadIdx.x; i < n; i += kThreads) cp_async16(smem_addr(smem + a.bytes_off) + i * 16, reinterpret_cast<const uint4*>(a.xcols) + i);
                for (int i = threadIdx.x; i < m; i += kThreads) cp_async16(smem_addr(smem + a.bytes_off) + (n + i) * 16, reinterpret_cast<const uint4*>(a.xmeta) + i);
                L.xbytes = smem + a.bytes_off;
                L.xmeta = reinterpret_cast<const int*>(smem + a.bytes_off + n * 16);
            }
            cp_commit();
        }
        const int entries = route(a, L);
        if constexpr (W::kBytes) {
            cp_wait<0>();
            __syncthreads();
        }
        constexpr int kDepth = depth<W, TILES>();
        const uint32_t ring = smem_addr(smem) + warp * kDepth * a.slot_bytes + lane * 16;
        {
            const Span s = span_of(a, entries * a.strips1, a.kb1, a.per_kb1);
            Fetcher<W, 1, TILES> f;
#pragma unroll 1
            for (int d = 0; d < kDepth; ++d) f.next(a, L, s, warp, lane, ring + d * a.slot_bytes, true, true);
            if (!s.whole) find_cuts(L, s, (int64_t)entries * a.strips1 * a.kb1);
            stream<W, 1, TILES>(a, L, s, f, smem);
            if (!s.whole) join<W, 1>(a, L, s);
        }
        grid_arrive(a.sync + 1);
        const Span s = span_of(a, a.strips2, entries * a.kb2, __frcp_rn((float)(entries * a.kb2)));
        Fetcher<W, 2, TILES> f, g;                           // ahead of the barrier the weights, behind it their columns
#pragma unroll 1
        for (int d = 0; d < kDepth; ++d) f.next(a, L, s, warp, lane, ring + d * a.slot_bytes, true, false);
        ok = grid_wait(a.sync + 1, a.sync + 3, a.polls, &flag);
        if (ok) {
            if (!W::kBytes) {
#pragma unroll 1
                for (int d = 0; d < kDepth; ++d) g.next(a, L, s, warp, lane, ring + d * a.slot_bytes, false, true);
            }
            if (!s.whole) find_cuts(L, s, (int64_t)a.strips2 * entries * a.kb2);
            stream<W, 2, TILES>(a, L, s, W::kBytes ? f : g, smem);
            if (!s.whole) join<W, 2>(a, L, s);
        }
        cp_wait<0>();
    }
    __syncthreads();
    if (threadIdx.x == 0 && atomicAdd(a.sync + 2, 1) == (int)gridDim.x - 1) a.sync[0] = a.sync[1] = a.sync[2] = 0;   // the last one out
}

// 16-bit matrices to units: a thread writes the 16 bytes one lane of Wide::unit reads.
__global__ void wide_pack_kernel(unsigned char* dst, const uint16_t* w, int rows, int cols, int strips, int blocks, int paired, int64_t n_units) {
    const int64_t stride = (int64_t)gridDim.x * blockDim.x;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n_units * 64; i += stride) {
        const int64_t unit = i >> 6;
        const int part = (int)(i & 63), lane = part & 31, slice = part >> 5, g = lane >> 2, t = lane & 3;
        const int block = (int)(unit % blocks);
        const int64_t ms = unit / blocks;
        const int c = block * 32 + 8 * t + 4 * slice;
        uint32_t v[4] = {0u, 0u, 0u, 0u};                     // registers of the operand: rows g, g + 8, g, g + 8; columns c, c, c + 2, c + 2
        for (int h = 0; h < 2; ++h) {
            const int r = strip_row(rows, paired, (int)(ms % strips), g, h);
            if (r < 0) continue;
            const uint16_t* p = w + (ms / strips * rows + r) * cols + c;
            for (int e = 0; e < 4; ++e)
                if (c + e < cols) v[h + (e & 2)] |= (uint32_t)p[e] << (16 * (e & 1));
        }
        *reinterpret_cast<uint4*>(dst + unit * 1024 + slice * 512 + lane * 16) = make_uint4(v[0], v[1], v[2], v[3]);
    }
}

__global__ void router_pack_kernel(float* dst, const void* r, int type, int E, int H, int ld) {
    for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < E * ld; i += gridDim.x * blockDim.x) {
        const int e = i / ld, c = i - e * ld;
        const int64_t at = (int64_t)e * H + c;
        dst[i] = c >= H ? 0.0f : type == PP_F32 ? static_cast<const float*>(r)[at]
                 : type == PP_F16 ? to_float(static_cast<const __half*>(r)[at]) : to_float(static_cast<const __nv_bfloat16*>(r)[at]);
    }
}

// The largest square of a row's norm among gate rows (most[0]) and up rows (most[1]) of all experts, rows that are not finite left
// out (what they give is not finite either); a warp to a row.  scales: of 4-bit codes, else binary16 weights.
__global__ void row_norms_kernel(unsigned long long* most, const void* w, const uint16_t* scales, const uint8_t* zeros, bool bf16_scales, int64_t rows,
                                 int F, int cols, int group) {
    const int lane = threadIdx.x & 31, groups = group ? (cols + group - 1) / group : 1;
    const int64_t code_ld = (cols + 1) / 2, step = (int64_t)gridDim.x * (blockDim.x >> 5);
    for (int64_t r = (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5); r < rows; r += step) {
        double sum = 0.0;
        for (int c = lane; c < cols; c += 32) {
            float v;
            if (scales) {
                const int64_t at = r * groups + (group ? c / group : 0);
                const uint16_t s = scales[at];
                const int q = static_cast<const uint8_t*>(w)[r * code_ld + c / 2] >> (4 * (c & 1)) & 15, z = zeros ? zeros[at] & 15 : 8;
                v = (float)(q - z) * (bf16_scales ? __uint_as_float((uint32_t)s << 16) : __half2float(__ushort_as_half(s)));
            } else {
                v = __half2float(static_cast<const __half*>(w)[r * cols + c]);
            }
            sum += (double)v * v;
        }
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == 0 && sum < INFINITY) atomicMax(most + (r % (2 * F) >= F), (unsigned long long)__double_as_longlong(sum));
    }
}

// The exponent of a power of two that no product of a gate row's and an up row's norm exceeds.
cudaError_t find_act_bound(pp_moe* L, const void* w, const void* scales, const void* zeros, int group, cudaStream_t stream) {
    unsigned long long* most = nullptr;
    double norms[2] = {0.0, 0.0};
    const int64_t rows = (int64_t)L->E * 2 * L->F;
    cudaError_t e = cudaMalloc(&most, sizeof(norms));
    if (e == cudaSuccess) e = cudaMemsetAsync(most, 0, sizeof(norms), stream);
    if (e == cudaSuccess) {
        row_norms_kernel<<<(unsigned)std::min<int64_t>((rows + 7) / 8, sm_count() * 16), 256, 0, stream>>>(
            most, w, static_cast<const uint16_t*>(scales), static_cast<const uint8_t*>(zeros), L->bf16_scales, rows, L->F, L->H, group);
        e = cudaGetLastError();
    }
    if (e == cudaSuccess) e = cudaMemcpyAsync(norms, most, sizeof(norms), cudaMemcpyDeviceToHost, stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize(stream);
    cudaFree(most);
    // (rounding of the sums in fp32 has room above the bound: 2^26 of 2^27)
    if (e == cudaSuccess) L->act_bound = norms[0] > 0.0 && norms[1] > 0.0 ? (int)std::ceil(0.5 * (std::log2(norms[0]) + std::log2(norms[1]))) : 0;
    return e;
}

cudaError_t launch_wide_pack(void* dst, const void* w, int count, int rows, int cols, bool paired, cudaStream_t stream) {
    const int strips = strips_of(rows, paired), blocks = (cols + 31) / 32;
    const int64_t n = (int64_t)count * strips * blocks;
    const unsigned grid = (unsigned)std::min<int64_t>((n * 64 + 255) / 256, sm_count() * 32);
    wide_pack_kernel<<<grid, 256, 0, stream>>>(static_cast<unsigned char*>(dst), static_cast<const uint16_t*>(w), rows, cols, strips, blocks, paired, n);
    return cudaGetLastError();
}

using Kernel = void (*)(const MoeArgs);
template <int TILES> Kernel pick_kernel(const pp_moe* L) {
    if (L->wtype == PP_BF16) return moe_kernel<Wide<true>, TILES>;
    if (L->wtype == PP_F16) return moe_kernel<Wide<false>, TILES>;
    if (L->sets == 4) return L->asym ? moe_kernel<Q4<4, true>, TILES> : moe_kernel<Q4<4, false>, TILES>;
    if (L->sets == 2) return L->asym ? moe_kernel<Q4<2, true>, TILES> : moe_kernel<Q4<2, false>, TILES>;
    return L->asym ? moe_kernel<Q4<1, true>, TILES> : moe_kernel<Q4<1, false>, TILES>;
}
// Tokens of an entry: what two tiles of columns hold, or what one does, two, where few experts have more than that (their
// weights are then read again, from L2).  16-bit experts, bound by HBM, take two while they have less than a token each on
// average (64 experts of 2048 x 1024, 8 a token: 4 tokens 61.7 us with two, 62.5 with five; 8 tokens 101.8 and 98.4); 4-bit
// experts, bound by the products, up to two tokens each (4 tokens 33.1 us with two, 38.7 with four, all that two tiles of four
// columns a token hold; 16 tokens, two each, 77.0 and 83.4; 8 experts of 4096 x 2048, three each 53.9 and 52.3, four each 67.1
// and 59.8).
int cap_of(int tokens, int top_k, int E, bool q4) {
    return (q4 ? tokens * top_k <= 2 * E : tokens * top_k < E) ? 8 / (q4 ? kByteCols : kActCols) : q4 ? kMaxCols / kByteCols : kMaxCap;
}
int tiles_of(int tokens, int cap) { return std::min(tokens, cap) * kActCols <= 8 ? 1 : 2; }

constexpr int kMaxSmem = 227 * 1024 - 384;       // beside the kernel's few static bytes

// Strips of a round and the shared memory: the most strips that fit, 32 at most.
size_t plan_smem(MoeArgs& a, int ring, int tiles, int meta) {
    size_t at = (size_t)kWarps * ring;
    a.list_off = (int)(at = (at + 127) / 128 * 128);
    at += list_bytes(a.T, a.E, a.top_k);
    a.scr_off = (int)at;
    at += (size_t)kWarps * 16 * 8 * tiles * 4;
    a.park_off = (int)at;
    for (a.round = 32, a.round_log2 = 5;; a.round /= 2, --a.round_log2) {
        const size_t total = at + (size_t)(a.round + kWarps) * 16 * std::max(a.cap, a.T) * 4;
        if (total > (size_t)kMaxSmem && a.round > 1) continue;
        const size_t bytes = meta ? (size_t)a.T * kByteCols * a.kpad1 + (size_t)a.T * kByteCols * a.kb1 * meta * 4 + 16 : 0;
        const bool fits = bytes && total + bytes <= (size_t)kMaxSmem;
        a.bytes_off = fits ? (int)total : 0;
        return total + (fits ? bytes : 0);
    }
}

size_t sync_bytes(int ctas) { return (4 + 2 * (size_t)ctas) * 4; }
template <typename T> bool alloc(T** p, size_t n) { return cudaMalloc(reinterpret_cast<void**>(p), n) == cudaSuccess; }

}  // namespace
}  // namespace pp

using namespace pp;

extern "C" pp_status_t pp_moe_destroy(pp_moe_t* L) {
    if (!L) return PP_ERR_INVALID_ARG;
    for (void* p : {static_cast<void*>(L->gate_up), static_cast<void*>(L->down), static_cast<void*>(L->gate_up_sets),
                    static_cast<void*>(L->down_sets), static_cast<void*>(L->router), static_cast<void*>(L->logits),
                    static_cast<void*>(L->xscale), static_cast<void*>(L->xcols), static_cast<void*>(L->acols), static_cast<void*>(L->xmeta), static_cast<void*>(L->parts), static_cast<void*>(L->sync)})
        cudaFree(p);
    delete L;
    return PP_OK;
}

// Everything but the experts' weights; wtype -1: 4-bit codes in groups.
static pp_status_t moe_new(pp_moe_t** out, int E, int H, int F, int top_k, int renorm, int max_tokens, const void* router, pp_dtype_t router_type,
                           int wtype, int group, bool asym, cudaStream_t s) {
    if (!out) return PP_ERR_INVALID_ARG;
    *out = nullptr;
    if (E < 1 || H < 1 || F < 1 || top_k < 1 || top_k > E || max_tokens < 1 || !router) return PP_ERR_INVALID_ARG;
    if (E > kMaxExperts || top_k > kMaxTopK || max_tokens > kMaxTokens || H > (1 << 16) || F > (1 << 16) || !is_float(router_type))
        return PP_ERR_UNSUPPORTED;
    if (!aligned_to(router, type_bytes(router_type))) return PP_ERR_INVALID_ARG;
    pp_moe* L = new (std::nothrow) pp_moe{};
    if (!L) return PP_ERR_ALLOC;
    L->E = E;
    L->H = H;
    L->F = F;
    L->top_k = top_k;
    L->renorm = renorm != 0;
    L->max_tokens = max_tokens;
    L->wtype = wtype;
    L->sets = wtype < 0 ? q4_sets(group) : 0;
    L->asym = asym;
    const int cols = wtype < 0 ? kQ4UnitCols : 32;
    L->strips1 = strips_of(2 * F, true);
    L->strips2 = strips_of(H, false);
    L->kb1 = (H + cols - 1) / cols;
    L->kb2 = (F + cols - 1) / cols;
    const size_t pairs = (size_t)max_tokens * top_k, ld = (size_t)(H + 3) / 4 * 4;
    const size_t units1 = (size_t)E * L->strips1 * L->kb1, units2 = (size_t)E * L->strips2 * L->kb2;
    const size_t set_bytes = wtype < 0 ? q4_set_bytes(L->sets, asym) : 0, abytes = pairs * kActCols * L->kb2 * cols * 2;
    pp_status_t st = PP_OK;
    // as many CTAs as the device holds at once, asked for with the most shared memory a call may take
    int device = 0, sms = 0;
    if (cudaGetDevice(&device) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess) st = PP_ERR_CUDA;
    for (Kernel kernel : {pick_kernel<1>(L), pick_kernel<2>(L)}) {
        int each = 0;
        if (st == PP_OK && (cudaFuncSetAttribute(reinterpret_cast<const void*>(kernel), cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem) != cudaSuccess ||
                            cudaOccupancyMaxActiveBlocksPerMultiprocessor(&each, kernel, kThreads, kMaxSmem) != cudaSuccess || each < 1)) st = PP_ERR_CUDA;
    }
    L->device = device;
    L->ctas = sms;
    if (st == PP_OK &&
        (!alloc(&L->gate_up, units1 * 1024) || !alloc(&L->down, units2 * 1024) ||
         (set_bytes && (!alloc(&L->gate_up_sets, units1 * set_bytes) || !alloc(&L->down_sets, units2 * set_bytes))) || !alloc(&L->router, ld * E * 4) ||
         !alloc(&L->logits, (size_t)max_tokens * E * kRouterParts * 4) || !alloc(&L->xscale, (size_t)max_tokens * 8) ||
         !alloc(&L->xcols, (size_t)max_tokens * 3 * L->kb1 * cols * 2) || !alloc(&L->acols, abytes) ||
         (wtype < 0 && !alloc(&L->xmeta, (size_t)max_tokens * kByteCols * L->kb1 * 32)) ||
         !alloc(&L->parts, (size_t)L->ctas * 2 * 16 * std::max(kMaxCap, max_tokens) * 4) || !alloc(&L->sync, sync_bytes(L->ctas)))) {
        st = PP_ERR_ALLOC;
    }
    if (st == PP_OK) {
        // act's columns past F are never written and stay zero
        if (cudaMemsetAsync(L->acols, 0, abytes, s) != cudaSuccess || cudaMemsetAsync(L->sync, 0, sync_bytes(L->ctas), s) != cudaSuccess) st = PP_ERR_CUDA;
        router_pack_kernel<<<sm_count(), 256, 0, s>>>(L->router, router, router_type, E, H, (int)ld);
        if (cudaGetLastError() != cudaSuccess) st = PP_ERR_CUDA;
    }
    if (st != PP_OK) {
        cudaGetLastError();
        pp_moe_destroy(L);
        return st;
    }
    *out = L;
    return PP_OK;
}

static pp_status_t moe_filled(pp_moe_t** out, cudaError_t e, cudaStream_t s) {
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    const pp_status_t st = status_of(e);
    if (st != PP_OK) {
        pp_moe_destroy(*out);
        *out = nullptr;
    }
    return st;
}

extern "C" pp_status_t pp_moe_create(pp_moe_t** out, int E, int H, int F, int top_k, int renormalize, int max_tokens, const void* router,
                                     pp_dtype_t router_type, const void* gate_up, const void* down, pp_dtype_t wtype, void* cuda_stream) {
    if (out) *out = nullptr;
    if (!gate_up || !down || !aligned_to(gate_up, 2) || !aligned_to(down, 2)) return PP_ERR_INVALID_ARG;
    if (!is_16bit(wtype)) return PP_ERR_UNSUPPORTED;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    const pp_status_t st = moe_new(out, E, H, F, top_k, renormalize, max_tokens, router, router_type, wtype, 0, false, s);
    if (st != PP_OK) return st;
    cudaError_t e = launch_wide_pack((*out)->gate_up, gate_up, E, 2 * F, H, true, s);
    if (e == cudaSuccess) e = launch_wide_pack((*out)->down, down, E, H, F, false, s);
    if (e == cudaSuccess && wtype == PP_F16) e = find_act_bound(*out, gate_up, nullptr, nullptr, 0, s);
    return moe_filled(out, e, s);
}

extern "C" pp_status_t pp_moe_create_q4(pp_moe_t** out, int E, int H, int F, int top_k, int renormalize, int max_tokens, const void* router,
                                        pp_dtype_t router_type, int group, const void* gate_up_codes, const void* gate_up_scales,
                                        const void* gate_up_zeros, const void* down_codes, const void* down_scales, const void* down_zeros,
                                        pp_dtype_t scale_type, void* cuda_stream) {
    if (out) *out = nullptr;
    if (!gate_up_codes || !gate_up_scales || !down_codes || !down_scales || (gate_up_zeros == nullptr) != (down_zeros == nullptr) || group < 0 ||
        !aligned_to(gate_up_scales, 2) || !aligned_to(down_scales, 2)) return PP_ERR_INVALID_ARG;
    if (!is_16bit(scale_type) || !q4_group_ok(group)) return PP_ERR_UNSUPPORTED;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    const pp_status_t st = moe_new(out, E, H, F, top_k, renormalize, max_tokens, router, router_type, -1, group, gate_up_zeros != nullptr, s);
    if (st != PP_OK) return st;
    (*out)->bf16_scales = scale_type == PP_BF16;
    cudaError_t e = launch_q4_pack((*out)->gate_up, (*out)->gate_up_sets, gate_up_codes, gate_up_scales, gate_up_zeros, E, 2 * F, H, group, true, s);
    if (e == cudaSuccess) e = launch_q4_pack((*out)->down, (*out)->down_sets, down_codes, down_scales, down_zeros, E, H, F, group, false, s);
    if (e == cudaSuccess) e = find_act_bound(*out, gate_up_codes, gate_up_scales, gate_up_zeros, group, s);
    return moe_filled(out, e, s);
}

extern "C" pp_status_t pp_moe_status(pp_moe_t* L, pp_status_t* status) {
    if (!L || !status) return PP_ERR_INVALID_ARG;
    // the layer's device, whichever is the caller's: the counters are cleared only when none of its kernels is on the way
    struct On {
        int before = -1;
        explicit On(int device) {
            int now = 0;
            if (cudaGetDevice(&now) == cudaSuccess && now != device && cudaSetDevice(device) == cudaSuccess) before = now;
        }
        ~On() {
            if (before >= 0) cudaSetDevice(before);
        }
    } on(L->device);
    int raised = 0;
    if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpy(&raised, L->sync + 3, 4, cudaMemcpyDeviceToHost) != cudaSuccess) return PP_ERR_CUDA;
    // a wait that gave up leaves divided strips with some of their CTAs counted and nobody to take the count back: the whole of
    // it starts anew (not at the kernel's end: ordering that behind the other CTAs' counts costs every call 0.7 us)
    if (raised && cudaMemset(L->sync, 0, sync_bytes(L->ctas)) != cudaSuccess) return PP_ERR_CUDA;
    *status = raised ? PP_ERR_TIMEOUT : PP_OK;
    return PP_OK;
}

extern "C" pp_status_t pp_moe_forward(pp_moe_t* L, const void* x, int64_t ldx, pp_dtype_t x_type, void* y, pp_dtype_t y_type, int tokens,
                                      int32_t* ids_out, float* gates_out, void* cuda_stream) {
    if (!L || !x || !y || x == y || tokens < 1 || tokens > L->max_tokens || (tokens > 1 && ldx < L->H)) return PP_ERR_INVALID_ARG;
    if (!is_float(x_type) || !is_float(y_type)) return PP_ERR_UNSUPPORTED;
    const int xb = type_bytes(x_type);
    if (!aligned_to(x, xb) || !aligned_to(y, type_bytes(y_type)) || !aligned_to(ids_out, 4) || !aligned_to(gates_out, 4)) return PP_ERR_INVALID_ARG;
    const bool q4 = L->wtype < 0;
    const int cols = q4 ? kQ4UnitCols : 32;
    MoeArgs a{};
    a.gate_up = L->gate_up;
    a.down = L->down;
    a.router = L->router;
    a.in.x = x;
    a.in.ld = ldx;
    a.in.type = x_type;
    a.in.cols = L->H;
    a.in.vec = aligned_to(x, 4 * xb) && (tokens == 1 || ldx % 4 == 0) && L->H % 4 == 0;
    a.logits = L->logits;
    a.xscale = L->xscale;
    a.xcols = L->xcols;
    a.acols = L->acols;
    a.xmeta = L->xmeta;
    a.sync = L->sync;
    a.y = y;
    a.ids = ids_out;
    a.gates = gates_out;
    a.y_type = y_type;
    a.T = tokens;
    a.E = L->E;
    a.H = L->H;
    a.top_k = L->top_k;
    a.renorm = L->renorm;
    a.act_bound = L->act_bound;
    a.strips1 = L->strips1;
    a.strips2 = L->strips2;
    a.kb1 = L->kb1;
    a.kb2 = L->kb2;
    a.kpad1 = L->kb1 * cols;
    a.kpad2 = L->kb2 * cols;
    a.router_ld = (L->H + 3) / 4 * 4;
    a.router_parts = std::max(1, std::min({kRouterParts, L->ctas * kWarps / (tokens * L->E), (L->H + 127) / 128}));
    a.router_cols = ((L->H + a.router_parts - 1) / a.router_parts + 127) / 128 * 128;
    a.cap = cap_of(tokens, L->top_k, L->E, q4);
    const int tiles = tiles_of(tokens, a.cap);
    const Kernel kernel = tiles == 1 ? pick_kernel<1>(L) : pick_kernel<2>(L);
    a.slot_bytes = 1024 + (q4 ? pad128(q4_set_bytes(L->sets, L->asym)) : 512 * tiles);
    const int ring = (!q4 && tiles == 2 ? 4 : 6) * a.slot_bytes;           // as depth() of the kernel
    a.gate_up_sets = L->gate_up_sets;
    a.down_sets = L->down_sets;
    a.cpt = q4 ? kByteCols : L->wtype == PP_BF16 ? (x_type == PP_BF16 ? 1 : x_type == PP_F16 ? 2 : 3) : (x_type == PP_F32 ? 2 : 1);
    a.bf16_scales = L->bf16_scales;
    a.polls = g_stream_wait_polls;
    a.parts = L->parts;
    a.per_expert = 1.0f / (float)L->strips1;
    a.per_entry = 1.0f / (float)L->kb2;
    a.per_kb1 = 1.0f / (float)L->kb1;
    a.per_cta = 1.0f / (float)L->ctas;
    a.per_cta64 = 1.0 / (double)L->ctas;
    a.per_cap = 1.0f / (float)a.cap;
    a.per_top_k = 1.0f / (float)L->top_k;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeCooperative;
    at[0].val.cooperative = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(L->ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = plan_smem(a, ring, tiles, !q4 ? 0 : L->sets == 1 ? 2 : L->sets == 2 ? 4 : 8);        // as kMeta
    cfg.stream = static_cast<cudaStream_t>(cuda_stream);
    cfg.attrs = at;
    cfg.numAttrs = 2;
    return status_of(cudaLaunchKernelEx(&cfg, kernel, a));
}
