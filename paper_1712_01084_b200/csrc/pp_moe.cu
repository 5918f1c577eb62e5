// A whole mixture-of-experts layer for a few tokens in one cooperative kernel.
//
//   l = R x (fp32),  the top_k largest (ties: the lowest index),  p = softmax(l), renormalised over the chosen or not
//   y = sum_j D_e(j) ( p_j * silu(G_e(j) x) * (U_e(j) x) )
//
// With a few tokens every chosen expert's weights are read once for one to a few columns, so the layer is bound by HBM
// on those weights, and for one token by the three steps that wait for one another:
//   step 0  the first CTAs turn the tokens into columns of the products' type, every warp of the grid takes (token,
//           expert) pairs of the router;                                                     -- grid barrier --
//   step 1  every CTA ranks the logits for itself (rank = how many are better: no sorting, no second barrier), lists the
//           experts that some token chose, and the grid streams their gate and up rows; eight rows of each share a
//           strip, so the CTA that finishes a strip has both halves of act = p silu(g) u;    -- grid barrier --
//   step 2  the grid streams the down rows; a strip of 16 rows of y collects all experts, so nothing is summed across
//           clusters.  The first of these weights are requested before the barrier.
// A cluster of S CTAs shares a run of strips and splits their columns; its partial sums meet in distributed shared
// memory.  Inside a CTA the units of a round of strips are dealt to the 16 warps in equal runs, each with a ring of
// asynchronous copies in flight.  All sums are taken in one fixed order.
//
// Columns.  Products take one 16-bit type, the weights' (binary16 for 4-bit codes).  An input that has more bits than
// one column holds is split over several: bf16 products take f16 in two and f32 in three columns; binary16 products take
// a token times the power of two that brings its largest magnitude to [2^13, 2^14), in one column for bf16 and two for
// f32.  act is f32 and always takes three: in bf16 these are its 24 bits; in binary16, where no scale is known before
// all of act is, they hold act * 2^-11, the rest * 2^-1 and the rest * 2^10, which together are act to 24 bits between
// 2^-11 and 2^27 and to an absolute 2^-35 below.
#include "pp_q4.cuh"

#include <algorithm>
#include <new>

namespace pp {
extern int g_stream_wait_polls;
}

struct pp_moe {
    int E, H, F, top_k, renorm, max_tokens, wtype, sets;      // wtype: PP_F16, PP_BF16 or -1 for 4-bit codes
    bool asym, bf16_scales;
    int strips1, strips2, kb1, kb2;
    int ctas[5];              // CTAs the device holds at once, for clusters of 1, 2 and 4
    unsigned char *gate_up, *down, *gate_up_sets, *down_sets;
    float *router, *logits, *xscale;
    uint16_t *xcols, *acols;
    int* sync;                // [0], [1] arrivals at the two barriers, [2] CTAs that are done, [3] status
};

namespace pp {
namespace {

constexpr int kWarps = 16, kThreads = kWarps * 32, kDepth = 6, kTiles = 2, kCols = 8 * kTiles;
constexpr int kMaxExperts = 256, kMaxTopK = 16, kMaxTokens = 32, kActCols = 3, kCap = kCols / kActCols;   // tokens of an entry
constexpr int kSpinPolls = 1 << 24;          // seconds; a barrier that is met never gets near it

struct MoeArgs {
    const unsigned char *gate_up, *down, *gate_up_sets, *down_sets;       // units, and their sets of 4-bit scales
    const float* router;
    XIn in;
    float *logits, *xscale;
    uint16_t *xcols, *acols;
    int* sync;
    void* y;
    int32_t* ids;
    float* gates;
    int y_type, T, E, H, top_k, renorm, strips1, strips2, kb1, kb2, kpad1, kpad2, router_ld, slot_bytes, cpt, bf16_scales, polls;
    int round1, round2;                      // strips of a round in steps 1 and 2
    int red_floats;                          // size of one of the two reduction buffers
    int list_off, scr_off, park_off, red_off;   // shared memory; the weight rings are at 0
};

// ---- weight formats: bytes and columns of a unit, and its product with the columns a lane reads ------------------
__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint4& a, uint32_t b0, uint32_t b1) {
    asm(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b0), "r"(b1));
}

template <bool BF16> struct Wide {           // 16-bit weights: 16 rows x 32 columns, two operand fragments of 512 bytes
    static constexpr int kUnitCols = 32, kSetBytes = 0;
    static constexpr bool kBf16 = BF16, kSwap = false;
    template <int NT, typename LoadX>
    static __device__ __forceinline__ void unit(float (&tot)[NT][4], const unsigned char* slot, int lane, bool, LoadX load_x) {
        const uint4 a = at<uint4>(slot + lane * 16), b = at<uint4>(slot + 512 + lane * 16);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const uint4 x = load_x(nt, 0);
            if (BF16) {
                mma_bf16(tot[nt], a, x.x, x.y);
                mma_bf16(tot[nt], b, x.z, x.w);
            } else {
                const uint32_t ar[4] = {a.x, a.y, a.z, a.w}, br[4] = {b.x, b.y, b.z, b.w};
                mma_f16(tot[nt], ar, x.x, x.y);
                mma_f16(tot[nt], br, x.z, x.w);
            }
        }
    }
};

template <int SETS, bool ASYM> struct Q4 {
    static constexpr int kUnitCols = kQ4UnitCols, kSetBytes = SETS * (ASYM ? 48 : 32);
    static constexpr bool kBf16 = false, kSwap = true;        // kSwap: columns 4i + 1 and 4i + 2 of the input change places
    template <int NT, typename LoadX>
    static __device__ __forceinline__ void unit(float (&tot)[NT][4], const unsigned char* slot, int lane, bool bf16_scales, LoadX load_x) {
        q4_unit_f16<NT, SETS, ASYM>(tot, slot, lane, bf16_scales, load_x);
    }
};

// ---- small helpers -----------------------------------------------------------------------------------------------
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
__device__ __forceinline__ uint32_t at_rank(uint32_t local, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(local), "r"(rank));
    return r;
}
__device__ __forceinline__ void st_cluster(uint32_t local, uint32_t rank, float v) {
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at_rank(local, rank)), "f"(v) : "memory");
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}
// All CTAs of the cluster, or of the block where it has none.
__device__ __forceinline__ void group_sync(int S) {
    if (S > 1) cluster_sync();
    else __syncthreads();
}

// Every CTA of the grid has arrived and what it wrote before is visible; false (in every CTA of the cluster alike) if the
// wait gave up.  One CTA of a cluster polls and tells the others through their shared memory (each barrier has a flag of
// its own there: a CTA that is slow to read the first must not find the second's answer).
__device__ __forceinline__ bool grid_barrier(int* counter, int* status, int S, int rank, int polls, int* flag) {
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        atomicAdd(counter, 1);
        if (rank == 0) {
            const int limit = polls > 0 ? polls : kSpinPolls;
            int seen = 0;
            for (int i = 0; i < limit; ++i) {
                asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(seen) : "l"(counter) : "memory");
                if (seen >= (int)gridDim.x) break;
            }
            const bool ok = seen >= (int)gridDim.x;
            if (!ok) *status = 1;
            *flag = ok;
            for (int r = 1; r < S; ++r)
                asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(at_rank(smem_addr(flag), r)), "r"(ok ? 1 : 0) : "memory");
        }
    }
    group_sync(S);
    return *flag != 0;
}

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

// Columns a token takes.
template <bool BF16, typename T> __host__ __device__ constexpr int columns() {
    return std::is_same_v<T, float> ? (BF16 ? 3 : 2) : BF16 && std::is_same_v<T, __half> ? 2 : 1;
}

// The power of two that brings a magnitude `most` to [2^13, 2^14), and its inverse; below 2^-113 the largest factor whose
// inverse is a normal number, infinities stay as they are.
__device__ __forceinline__ void token_scale(float most, float& up, float& down) {
    uint32_t e = __float_as_uint(most) >> 23;
    e = e >= 255u ? 140u : e < 14u ? 14u : e;
    up = __uint_as_float((267u - e) << 23);
    down = __uint_as_float((e - 13u) << 23);
}

// ---- step 0 ------------------------------------------------------------------------------------------------------
// One CTA turns a token into columns.
template <class W, typename T> __device__ void token_columns(const MoeArgs& a, int token, float* part) {
    constexpr bool BF16 = W::kBf16;
    constexpr int cpt = columns<BF16, T>();
    const T* x = static_cast<const T*>(a.in.x) + (int64_t)token * a.in.ld;
    float up = 1.0f, down = 1.0f;
    if (!BF16 && !std::is_same_v<T, __half>) {
        float most = 0.0f;
        for (int c = threadIdx.x * 4; c < a.H; c += kThreads * 4) {
            const Pack<T, 4> v = load_four(x, c, a.H, a.in.vec != 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) most = fmaxf(most, fabsf(to_float(v.v[i])));
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
        __syncthreads();                                     // an earlier token's values have been read
        if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = most;
        __syncthreads();
        most = part[threadIdx.x & (kWarps - 1)];
#pragma unroll
        for (int o = kWarps / 2; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
        token_scale(most, up, down);
    }
    uint16_t* dst = a.xcols + (int64_t)token * cpt * a.kpad1;
    for (int c = threadIdx.x * 4; c < a.kpad1; c += kThreads * 4) {       // zeros up to the padded length
        const Pack<T, 4> v = load_four(x, c, a.H, a.in.vec != 0);
        Pack<uint16_t, 4> bits[cpt];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float rest = to_float(v.v[i]) * up;
#pragma unroll
            for (int k = 0; k < cpt; ++k) rest -= round16<BF16>(rest, bits[k].v[W::kSwap && (i == 1 || i == 2) ? 3 - i : i]);
        }
#pragma unroll
        for (int k = 0; k < cpt; ++k) *reinterpret_cast<Pack<uint16_t, 4>*>(dst + (int64_t)k * a.kpad1 + c) = bits[k];
    }
    if (threadIdx.x == 0) a.xscale[token] = down;
}

// A warp's logit of one (token, expert); what cannot be compared ranks last.
template <typename T> __device__ __forceinline__ void router_logit(const MoeArgs& a, int token, int expert) {
    const int lane = threadIdx.x & 31;
    const float* r = a.router + (int64_t)expert * a.router_ld;
    const T* row = static_cast<const T*>(a.in.x) + (int64_t)token * a.in.ld;
    float sum = 0.0f;
    for (int c0 = lane * 4; c0 < a.H; c0 += 1024) {
        Pack<T, 4> x[8];
        float4 w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int c = c0 + i * 128;
            if (c >= a.H) break;
            x[i] = load_four(row, c, a.H, a.in.vec != 0);
            w[i] = __ldg(reinterpret_cast<const float4*>(r + c));
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (c0 + i * 128 >= a.H) break;
            sum = fmaf(to_float(x[i].v[0]), w[i].x, sum);
            sum = fmaf(to_float(x[i].v[1]), w[i].y, sum);
            sum = fmaf(to_float(x[i].v[2]), w[i].z, sum);
            sum = fmaf(to_float(x[i].v[3]), w[i].w, sum);
        }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) a.logits[token * a.E + expert] = sum == sum ? sum : -INFINITY;
}

template <class W, typename T> __device__ __forceinline__ void step0(const MoeArgs& a, float* part) {
    const int warp = threadIdx.x >> 5;
    for (int t = blockIdx.x; t < a.T; t += gridDim.x) token_columns<W, T>(a, t, part);
    for (int i = warp * gridDim.x + (gridDim.x - 1 - blockIdx.x); i < a.T * a.E; i += kWarps * gridDim.x) router_logit<T>(a, i / a.E, i % a.E);
}

// ---- routing, by every CTA for itself ----------------------------------------------------------------------------
struct Lists {
    int4* entry;         // {expert, first pair, pairs, 0}: an expert and up to kCap of its tokens
    int* pair_token;     // pairs (token, expert) in the order of the experts
    float* pair_gate;
    float* gate;         // [T][top_k]
    int* sums;           // scratch of the scan
    uint8_t* slot;       // [T][E]: which of the token's choices the expert is, 255 none
};
__host__ __device__ inline int list_bytes(int T, int E, int top_k) { return (T * top_k * (16 + 4 + 4 + 4) + 64 + T * E + 127) / 128 * 128; }
__device__ __forceinline__ Lists lists_at(unsigned char* p, int T, int top_k) {
    Lists L;
    const int n = T * top_k;
    L.entry = reinterpret_cast<int4*>(p);
    L.pair_token = reinterpret_cast<int*>(L.entry + n);
    L.pair_gate = reinterpret_cast<float*>(L.pair_token + n);
    L.gate = L.pair_gate + n;
    L.sums = reinterpret_cast<int*>(L.gate + n);
    L.slot = reinterpret_cast<uint8_t*>(L.sums + 16);
    return L;
}

__device__ int route(const MoeArgs& a, const Lists& L) {                   // the number of entries
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    for (int i = tid; i < a.T * a.E; i += kThreads) {
        const int t = i / a.E, e = i - t * a.E;
        const float* row = a.logits + t * a.E;
        const float l = row[e];
        int rank = 0;
#pragma unroll 8
        for (int j = 0; j < a.E; ++j) rank += row[j] > l || (row[j] == l && j < e);
        L.slot[i] = rank < a.top_k ? (uint8_t)rank : (uint8_t)255;
    }
    __syncthreads();
    for (int t = warp; t < a.T; t += kWarps) {
        const float* row = a.logits + t * a.E;
        float most = -INFINITY, sum = 0.0f;
        for (int e = lane; e < a.E; e += 32) most = fmaxf(most, row[e]);
#pragma unroll
        for (int o = 16; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
        for (int e = lane; e < a.E; e += 32)
            if (!a.renorm || L.slot[t * a.E + e] != 255) sum += expf(row[e] - most);
#pragma unroll
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        for (int e = lane; e < a.E; e += 32) {
            const int slot = L.slot[t * a.E + e];
            if (slot == 255) continue;
            const float p = expf(row[e] - most) / sum;
            L.gate[t * a.top_k + slot] = p;
            if (blockIdx.x == 0) {
                if (a.ids) a.ids[t * a.top_k + slot] = e;
                if (a.gates) a.gates[t * a.top_k + slot] = p;
            }
        }
    }
    // where each expert's pairs and entries start: both counts in one scan (neither exceeds 512)
    int n = 0;
    if (tid < a.E)
        for (int t = 0; t < a.T; ++t) n += L.slot[t * a.E + tid] != 255;
    int both = n | ((n + kCap - 1) / kCap) << 16;
    const int mine = both;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, both, o);
        if (lane >= o) both += v;
    }
    if (lane == 31) L.sums[warp] = both;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) before += L.sums[w];
        all += L.sums[w];
    }
    before += both - mine;
    if (n) {
        const int first = before & 0xffff, entry = before >> 16;
        for (int i = 0; i * kCap < n; ++i) L.entry[entry + i] = make_int4(tid, first + i * kCap, min(kCap, n - i * kCap), 0);
        int p = first;
        for (int t = 0; t < a.T; ++t) {
            const int slot = L.slot[t * a.E + tid];
            if (slot == 255) continue;
            L.pair_token[p] = t;
            L.pair_gate[p++] = L.gate[t * a.top_k + slot];
        }
    }
    __syncthreads();
    return all >> 16;
}

// ---- steps 1 and 2: the stream of weights ------------------------------------------------------------------------
// What one CTA does in a step: strips first .. first + count of its cluster, `round` at a time, and of each strip the
// blocks v0 .. v0 + nv.  In step 1 a strip belongs to one entry and its blocks are the columns of x; in step 2 a strip is
// 16 rows of y and its blocks are the entries' columns of act, one entry after another.
struct Span { int first, count, round, v0, nv; };
struct Run { const unsigned char *unit, *sets; int left, ls, entry, kb; };        // units that lie one after another

template <class W, int STEP> __device__ __forceinline__ void locate(const MoeArgs& a, const Lists& L, const Span& s, int round, int u, Run& r) {
    r.ls = u / s.nv;
    const int v = s.v0 + u - r.ls * s.nv;
    int strip = s.first + round * s.round + r.ls;
    if (STEP == 1) {
        r.entry = strip / a.strips1;
        strip -= r.entry * a.strips1;
        r.kb = v;
        r.left = s.v0 + s.nv - v;
    } else {
        r.entry = v / a.kb2;
        r.kb = v - r.entry * a.kb2;
        r.left = min(a.kb2 - r.kb, s.v0 + s.nv - v);
    }
    const int64_t at = ((int64_t)L.entry[r.entry].x * (STEP == 1 ? a.strips1 : a.strips2) + strip) * (STEP == 1 ? a.kb1 : a.kb2) + r.kb;
    r.unit = (STEP == 1 ? a.gate_up : a.down) + at * 1024;
    r.sets = (STEP == 1 ? a.gate_up_sets : a.down_sets) + at * W::kSetBytes;
}

// This warp's units of a round.
__device__ __forceinline__ void warp_range(const Span& s, int round, int warp, int& u0, int& u1) {
    const int U = min(s.round, s.count - round * s.round) * s.nv;
    u0 = (int)((int64_t)U * warp / kWarps);
    u1 = (int)((int64_t)U * (warp + 1) / kWarps);
}

template <class W, int STEP> struct Fetcher {
    int round = -1, u = 0, u1 = 0;
    Run run;
    __device__ __forceinline__ void next(const MoeArgs& a, const Lists& L, const Span& s, int rounds, int warp, int lane, uint32_t slot) {
        while (u == u1 && round < rounds) {
            if (++round < rounds) warp_range(s, round, warp, u, u1);
            run.left = 0;
        }
        if (u < u1) {
            if (run.left == 0) locate<W, STEP>(a, L, s, round, u, run);
            unit_fetch(slot, run.unit, run.sets, lane, W::kSetBytes / 16);
            run.unit += 1024;
            run.sets += W::kSetBytes;
            --run.left;
            ++u;
        }
        cp_commit();
    }
};

template <class W, int STEP>
__device__ __forceinline__ void stream(const MoeArgs& a, const Lists& L, const Span& s, Fetcher<W, STEP>& f, int rounds, unsigned char* smem, int S,
                                       int rank, int& buffer) {
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int cpt = STEP == 1 ? a.cpt : kActCols, width = STEP == 1 ? kCap : a.T, kpad = STEP == 1 ? a.kpad1 : a.kpad2;
    const uint16_t* cols = STEP == 1 ? a.xcols : a.acols;
    unsigned char* ring = smem + warp * kDepth * a.slot_bytes;
    float* scr = reinterpret_cast<float*>(smem + a.scr_off) + warp * 16 * kCols;
    float* park = reinterpret_cast<float*>(smem + a.park_off);
    int slot = 0;
    for (int round = 0; round < rounds; ++round) {
        const int rs = min(s.round, s.count - round * s.round), U = rs * s.nv;
        int u0, u1, strip = -1, tiles = 1;
        warp_range(s, round, warp, u0, u1);
        Run run;
        run.left = 0;
        const uint16_t* from[kTiles] = {};
        int4 entry = make_int4(0, 0, 0, 0);
        float tot[kTiles][4] = {};
        for (int u = u0; u < u1; ++u) {
            if (run.left == 0) {
                locate<W, STEP>(a, L, s, round, u, run);
                entry = L.entry[run.entry];
                tiles = (entry.z * cpt + 7) / 8;
#pragma unroll
                for (int nt = 0; nt < kTiles; ++nt) {
                    const int c = nt * 8 + g, p = entry.y + min(c / cpt, entry.z - 1);       // columns past the last repeat one
                    const int row = (STEP == 1 ? L.pair_token[p] : p) * cpt + c % cpt;
                    from[nt] = cols + (int64_t)row * kpad + run.kb * W::kUnitCols + t * 8;
                }
                if (STEP == 2 && run.ls != strip) {            // a new strip's sums of this warp
                    strip = run.ls;
                    for (int i = lane; i < 16 * width; i += 32) park[(warp + strip) * 16 * width + i] = 0.0f;
                }
            }
            cp_wait<kDepth - 1>();
            __syncwarp();
            const auto load_x = [&](int nt, int j) { return *reinterpret_cast<const uint4*>(from[nt] + j * 32); };
            unsigned char* at = ring + slot * a.slot_bytes;
            if (tiles == 1) W::template unit<1>(reinterpret_cast<float(&)[1][4]>(tot), at, lane, a.bf16_scales != 0, load_x);
            else W::template unit<kTiles>(tot, at, lane, a.bf16_scales != 0, load_x);
#pragma unroll
            for (int nt = 0; nt < kTiles; ++nt) from[nt] += W::kUnitCols;
            __syncwarp();
            f.next(a, L, s, rounds, warp, lane, smem_addr(at));
            if (++slot == kDepth) slot = 0;
            if (--run.left == 0 || u + 1 == u1) {
                // add a token's columns and park the sums: piece (warp, strip) has slot warp + strip
#pragma unroll
                for (int nt = 0; nt < kTiles; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        scr[(g + (i >> 1) * 8) * kCols + nt * 8 + 2 * t + (i & 1)] = tot[nt][i];
                        tot[nt][i] = 0.0f;
                    }
                __syncwarp();
                float* tile = park + (warp + run.ls) * 16 * width;
                for (int i = lane; i < 16 * entry.z; i += 32) {
                    const int row = i / entry.z, pl = i - row * entry.z;
                    const float* c = scr + row * kCols + pl * cpt;
                    if (STEP == 1) {
                        float v = c[0];
                        for (int k = 1; k < cpt; ++k) v += c[k];
                        tile[row * width + pl] = v;
                    } else {
                        const float v = W::kBf16 ? c[0] + c[1] + c[2] : fmaf(c[0], 0x1p11f, fmaf(c[1], 2.0f, c[2] * 0x1p-10f));
                        tile[row * width + L.pair_token[entry.y + pl]] += v;
                    }
                }
                __syncwarp();
            }
        }
        __syncthreads();

        // the pieces of a row in the order of the warps; each CTA of the cluster finishes an equal part of the results
        const int outs = rs * (STEP == 1 ? 8 * kCap : 16 * a.T), share = (outs + S - 1) / S;
        float* red = reinterpret_cast<float*>(smem + a.red_off) + buffer * a.red_floats;
        buffer ^= 1;
        const auto pieces = [&](int ls, int at) {
            float v = 0.0f;
            if (U) {
                const int w_lo = (kWarps * (ls * s.nv + 1) - 1) / U, w_hi = (kWarps * (ls * s.nv + s.nv) - 1) / U;
                for (int w = w_lo; w <= w_hi; ++w)
                    if ((int)((int64_t)U * w / kWarps) < (int)((int64_t)U * (w + 1) / kWarps)) v += park[(w + ls) * 16 * width + at];
            }
            return v;
        };
        for (int o = tid; o < outs; o += kThreads) {
            const int owner = o / share, at = rank * share + o - owner * share;
            if (STEP == 1) {
                const int ls = o / (8 * kCap), r = o - ls * 8 * kCap, pl = r % kCap;
                if (pl >= L.entry[(s.first + round * s.round + ls) / a.strips1].z) continue;
                const float gate = pieces(ls, r), up = pieces(ls, r + 8 * kCap);
                if (S > 1) {
                    st_cluster(smem_addr(red + 2 * at), owner, gate);
                    st_cluster(smem_addr(red + 2 * at + 1), owner, up);
                } else {
                    red[2 * at] = gate;
                    red[2 * at + 1] = up;
                }
            } else {
                const int token = o / (rs * 16), r = o - token * rs * 16;
                const float v = pieces(r >> 4, (r & 15) * width + token);
                if (S > 1) st_cluster(smem_addr(red + at), owner, v);
                else red[at] = v;
            }
        }
        group_sync(S);
        const int first = rank * share, last = min(outs, first + share);
        for (int o = first + tid; o < last; o += kThreads) {
            if (STEP == 1) {
                const int ls = o / (8 * kCap), r = o - ls * 8 * kCap, pl = r % kCap;
                const int strip_all = s.first + round * s.round + ls, en = strip_all / a.strips1;
                const int4 e = L.entry[en];
                if (pl >= e.z) continue;
                float gate = 0.0f, up = 0.0f;
                for (int q = 0; q < S; ++q) {
                    gate += red[2 * (q * share + o - first)];
                    up += red[2 * (q * share + o - first) + 1];
                }
                const int p = e.y + pl, row = (strip_all - en * a.strips1) * 8 + r / kCap;
                const float scale = __ldcg(a.xscale + L.pair_token[p]);
                gate *= scale;
                up *= scale;
                const float act = L.pair_gate[p] * (gate / (1.0f + expf(-gate)) * up);
                const int at = W::kSwap && ((row & 3) == 1 || (row & 3) == 2) ? row ^ 3 : row;
                split_act<W::kBf16>(act, a.acols + (int64_t)p * kActCols * a.kpad2 + at, a.kpad2);
            } else {
                const int token = o / (rs * 16), m = (s.first + round * s.round) * 16 + o - token * rs * 16;
                if (m >= a.H) continue;
                float v = 0.0f;
                for (int q = 0; q < S; ++q) v += red[q * share + o - first];
                store_y(a.y, (int64_t)token * a.H + m, a.y_type, v);
            }
        }
    }
}

template <class W> __global__ void __launch_bounds__(kThreads, 1) moe_kernel(const MoeArgs a) {
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ float part[kWarps];
    __shared__ int flag[2];
    const int S = (int)cluster_size(), rank = (int)cluster_rank(), clusters = gridDim.x / S, cl = blockIdx.x / S;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const Lists L = lists_at(smem + a.list_off, a.T, a.top_k);
    if (S > 1) asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
    pdl_release();
    pdl_wait();

    if (a.in.type == PP_BF16) step0<W, __nv_bfloat16>(a, part);
    else if (a.in.type == PP_F16) step0<W, __half>(a, part);
    else step0<W, float>(a, part);
    if (S > 1) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");     // the cluster's other CTAs have started
    bool ok = grid_barrier(a.sync, a.sync + 3, S, rank, a.polls, flag);
    if (ok) {
        const int entries = route(a, L);
        const uint32_t ring = smem_addr(smem) + (uint32_t)(warp * kDepth * a.slot_bytes);
        int buffer = 0;
        Span s;
        const int64_t strips = (int64_t)entries * a.strips1;
        s.first = (int)(strips * cl / clusters);
        s.count = (int)(strips * (cl + 1) / clusters) - s.first;
        s.round = a.round1;
        s.v0 = a.kb1 * rank / S;
        s.nv = a.kb1 * (rank + 1) / S - s.v0;
        {
            Fetcher<W, 1> f;
            const int rounds = (s.count + s.round - 1) / s.round;
            for (int d = 0; d < kDepth; ++d) f.next(a, L, s, rounds, warp, lane, ring + d * a.slot_bytes);
            stream<W, 1>(a, L, s, f, rounds, smem, S, rank, buffer);
        }
        s.first = a.strips2 * cl / clusters;
        s.count = a.strips2 * (cl + 1) / clusters - s.first;
        s.round = a.round2;
        s.v0 = entries * a.kb2 * rank / S;
        s.nv = entries * a.kb2 * (rank + 1) / S - s.v0;
        Fetcher<W, 2> f;
        const int rounds = (s.count + s.round - 1) / s.round;
        for (int d = 0; d < kDepth; ++d) f.next(a, L, s, rounds, warp, lane, ring + d * a.slot_bytes);
        ok = grid_barrier(a.sync + 1, a.sync + 3, S, rank, a.polls, flag + 1);
        if (ok) stream<W, 2>(a, L, s, f, rounds, smem, S, rank, buffer);
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

cudaError_t launch_wide_pack(void* dst, const void* w, int count, int rows, int cols, bool paired, cudaStream_t stream) {
    const int strips = strips_of(rows, paired), blocks = (cols + 31) / 32;
    const int64_t n = (int64_t)count * strips * blocks;
    const unsigned grid = (unsigned)std::min<int64_t>((n * 64 + 255) / 256, 148 * 32);
    wide_pack_kernel<<<grid, 256, 0, stream>>>(static_cast<unsigned char*>(dst), static_cast<const uint16_t*>(w), rows, cols, strips, blocks, paired, n);
    return cudaGetLastError();
}

using Kernel = void (*)(const MoeArgs);
Kernel pick_kernel(const pp_moe* L) {
    if (L->wtype == PP_BF16) return moe_kernel<Wide<true>>;
    if (L->wtype == PP_F16) return moe_kernel<Wide<false>>;
    if (L->sets == 4) return L->asym ? moe_kernel<Q4<4, true>> : moe_kernel<Q4<4, false>>;
    if (L->sets == 2) return L->asym ? moe_kernel<Q4<2, true>> : moe_kernel<Q4<2, false>>;
    return L->asym ? moe_kernel<Q4<1, true>> : moe_kernel<Q4<1, false>>;
}

constexpr int kMaxSmem = 227 * 1024 - 256;       // beside the kernel's few static bytes

// Strips of a round and the shared memory they take; the most strips that fit, 16 at most (one to a warp).
size_t plan_smem(MoeArgs& a, int S) {
    size_t at = (size_t)kWarps * kDepth * a.slot_bytes;
    a.list_off = (int)(at = (at + 127) / 128 * 128);
    at += list_bytes(a.T, a.E, a.top_k);
    a.scr_off = (int)at;
    at += (size_t)kWarps * 16 * kCols * 4;
    a.park_off = (int)at;
    for (int R = 16;; R /= 2) {
        a.round1 = a.round2 = R;
        const size_t park = (size_t)(R + kWarps) * 16 * std::max(kCap, a.T) * 4;
        a.red_floats = std::max(R * 8 * kCap + S, R * 8 * a.T + S) * 2;
        a.red_off = (int)(a.park_off + park);
        const size_t total = a.red_off + (size_t)a.red_floats * 8;
        if (total <= (size_t)kMaxSmem || R == 1) return total;
    }
}

// Resident CTAs of a cooperative launch with clusters of S, 0 if none.
int resident(Kernel k, int S, size_t smem) {
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = (unsigned)S;
    at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(S);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, k, &cfg) != cudaSuccess) {
        cudaGetLastError();
        return 0;
    }
    return n * S;
}

template <typename T> bool alloc(T** p, size_t n) { return cudaMalloc(reinterpret_cast<void**>(p), n) == cudaSuccess; }

}  // namespace
}  // namespace pp

using namespace pp;

extern "C" pp_status_t pp_moe_destroy(pp_moe_t* L) {
    if (!L) return PP_ERR_INVALID_ARG;
    for (void* p : {static_cast<void*>(L->gate_up), static_cast<void*>(L->down), static_cast<void*>(L->gate_up_sets),
                    static_cast<void*>(L->down_sets), static_cast<void*>(L->router), static_cast<void*>(L->logits),
                    static_cast<void*>(L->xscale), static_cast<void*>(L->xcols), static_cast<void*>(L->acols), static_cast<void*>(L->sync)})
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
    const size_t abytes = pairs * kActCols * L->kb2 * cols * 2;
    pp_status_t st = PP_OK;
    const size_t units1 = (size_t)E * L->strips1 * L->kb1, units2 = (size_t)E * L->strips2 * L->kb2, set_bytes = wtype < 0 ? q4_set_bytes(L->sets, asym) : 0;
    if (!alloc(&L->gate_up, units1 * 1024) || !alloc(&L->down, units2 * 1024) ||
        (set_bytes && (!alloc(&L->gate_up_sets, units1 * set_bytes) || !alloc(&L->down_sets, units2 * set_bytes))) || !alloc(&L->router, ld * E * 4) ||
        !alloc(&L->logits, (size_t)max_tokens * E * 4) || !alloc(&L->xscale, (size_t)max_tokens * 4) ||
        !alloc(&L->xcols, (size_t)max_tokens * 3 * L->kb1 * cols * 2) || !alloc(&L->acols, abytes) || !alloc(&L->sync, 16)) {
        cudaGetLastError();
        st = PP_ERR_ALLOC;
    }
    if (st == PP_OK) {
        // act's columns past F are never written and stay zero
        if (cudaMemsetAsync(L->acols, 0, abytes, s) != cudaSuccess || cudaMemsetAsync(L->sync, 0, 16, s) != cudaSuccess) st = PP_ERR_CUDA;
        router_pack_kernel<<<148, 256, 0, s>>>(L->router, router, router_type, E, H, (int)ld);
        if (cudaGetLastError() != cudaSuccess ||
            cudaFuncSetAttribute(reinterpret_cast<const void*>(pick_kernel(L)), cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem) != cudaSuccess)
            st = PP_ERR_CUDA;
    }
    // one CTA to an SM, whatever the call's shared memory: asked for the most
    for (int S = 1; S <= 4 && st == PP_OK; S *= 2) L->ctas[S] = resident(pick_kernel(L), S, kMaxSmem);
    if (st == PP_OK && L->ctas[1] < 1) st = PP_ERR_CUDA;
    if (st != PP_OK) {
        pp_moe_destroy(L);
        return st;
    }
    *out = L;
    return PP_OK;
}

static pp_status_t moe_filled(pp_moe_t** out, cudaError_t e, cudaStream_t s) {
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    if (e == cudaSuccess) return PP_OK;
    pp_moe_destroy(*out);
    *out = nullptr;
    return PP_ERR_CUDA;
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
    return moe_filled(out, e, s);
}

extern "C" pp_status_t pp_moe_status(pp_moe_t* L, pp_status_t* status) {
    if (!L || !status) return PP_ERR_INVALID_ARG;
    int raised = 0;
    if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpy(&raised, L->sync + 3, 4, cudaMemcpyDeviceToHost) != cudaSuccess) return PP_ERR_CUDA;
    if (raised && cudaMemset(L->sync + 3, 0, 4) != cudaSuccess) return PP_ERR_CUDA;
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
    a.in.vec = aligned_to(x, 4 * xb) && (tokens == 1 || ldx % 4 == 0);
    a.logits = L->logits;
    a.xscale = L->xscale;
    a.xcols = L->xcols;
    a.acols = L->acols;
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
    a.strips1 = L->strips1;
    a.strips2 = L->strips2;
    a.kb1 = L->kb1;
    a.kb2 = L->kb2;
    a.kpad1 = L->kb1 * cols;
    a.kpad2 = L->kb2 * cols;
    a.router_ld = (L->H + 3) / 4 * 4;
    a.slot_bytes = 1024 + (q4 ? (q4_set_bytes(L->sets, L->asym) + 127) / 128 * 128 : 0);      // slots start on 128 bytes
    a.gate_up_sets = L->gate_up_sets;
    a.down_sets = L->down_sets;
    a.cpt = L->wtype == PP_BF16 ? (x_type == PP_BF16 ? 1 : x_type == PP_F16 ? 2 : 3) : (x_type == PP_F32 ? 2 : 1);
    a.bf16_scales = L->bf16_scales;
    a.polls = g_stream_wait_polls;
    // cluster size: fewest blocks on the busiest CTA, for the experts the tokens reach at most
    const int64_t experts = std::min<int64_t>(L->E, (int64_t)tokens * L->top_k);
    int best = 0;
    int64_t least = 0;
    for (int S = 1; S <= 4; S *= 2) {
        const int64_t n = L->ctas[S] / S;
        if (n < 1) continue;
        const int64_t cost = (experts * L->strips1 + n - 1) / n * ((L->kb1 + S - 1) / S) + (L->strips2 + n - 1) / n * ((experts * L->kb2 + S - 1) / S);
        if (!best || cost < least) best = S, least = cost;
    }
    const size_t smem = plan_smem(a, best);
    cudaLaunchAttribute at[3];
    at[0].id = cudaLaunchAttributeCooperative;
    at[0].val.cooperative = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    at[2].id = cudaLaunchAttributeClusterDimension;
    at[2].val.clusterDim.x = (unsigned)best;
    at[2].val.clusterDim.y = at[2].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(L->ctas[best]);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = static_cast<cudaStream_t>(cuda_stream);
    cfg.attrs = at;
    cfg.numAttrs = best > 1 ? 3 : 2;
    if (cudaLaunchKernelEx(&cfg, pick_kernel(L), a) == cudaSuccess) return PP_OK;
    cudaGetLastError();
    return PP_ERR_CUDA;
}
