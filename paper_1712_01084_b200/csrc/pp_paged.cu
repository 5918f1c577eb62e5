// Paged key-value cache: the plan of a step (pages and slots of the new tokens) and the append of their keys and values with
// rotary embedding.
//
// Plan.  A request that holds h tokens and gets a more needs the pages ceil(h / p) .. ceil((h + a) / p); where they start in the
// free list is an exclusive sum over the requests before it, as is the first row of its tokens.  Every CTA makes both sums
// for all requests (a few thousand additions in shared memory, cheaper than a second launch that would wait for a first),
// then takes its share of the pages and of the rows: a binary search for the request, and for a row its page from the free list
// where it is a new one, else from the table, whose old entries nobody writes.  All latency: 2.1 us for one request, 3.2 for 256
// (4.9 with a warp to a request's pages and four rows to a thread), 5.9 for 48 prompts with 200,000 tokens.
//
// Append.  All bandwidth for many tokens, all latency for few.  Both elements of a pair are in one lane and take the same sine.  The
// angle is a product in 64 bits, brought into a turn there: position 10^6 leaves a 32-bit angle 2^-5 of a radian.  16384 tokens
// of 64 + 2 x 8 heads of 128, bf16: 108 us, 6.2 TB/s; one token 2.1 us.
#include "pp_internal.h"
#include "pp_paged.cuh"

namespace pp {
namespace {

// -------------------------------------------------------------------------------------------------------- plan
constexpr int kPlanThreads = 256, kMaxRequests = 8192;

struct PlanArgs {
    const int32_t *lengths, *added, *free_pages, *taken;
    int32_t* table;
    int64_t* slots;
    int32_t *positions, *starts, *lengths_out, *taken_out;
    int64_t ld_table;
    int width, n_free, requests, page_size, rows, capacity;
    Divisor page;
    bool wide;                                               // slots and positions start on 16 bytes
    bool rows_too, state_too;                                // what this launch writes: rows, starts and table; lengths_out and taken_out
};

__device__ __forceinline__ int sat32(int64_t v) { return v > INT32_MAX ? INT32_MAX : (int)v; }

// kPlanRows: neighbouring rows of a thread.
template <int kPlanRows> __global__ void __launch_bounds__(kPlanThreads) plan_kernel(const PlanArgs a) {
    extern __shared__ int32_t plan_smem[];
    int32_t* starts = plan_smem;                             // [requests + 1]
    int32_t* have = starts + a.requests + 1;                 // [requests]
    int32_t* base = have + a.requests;                       // [requests]: pages that requests before this one need
    __shared__ int64_t warp_pages[8], warp_rows[8];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    pdl_release();
    pdl_wait();
    const int each = (a.requests + kPlanThreads - 1) / kPlanThreads, r0 = min(tid * each, a.requests), r1 = min(r0 + each, a.requests);
    const int64_t taken = *a.taken;
    int64_t pages = 0, rows = 0;
    for (int r = r0; r < r1; ++r) {
        const int h = min(max(a.lengths[r], 0), a.capacity), add = max(a.added[r], 0);
        const int total = (int)min((int64_t)h + add, (int64_t)a.capacity);
        have[r] = h;
        base[r] = (int)(a.page.of(total + a.page_size - 1) - a.page.of(h + a.page_size - 1));
        starts[r] = add;
        pages += base[r];
        rows += add;
    }
    int64_t before_pages = pages, before_rows = rows;        // inclusive, over the lanes, then over the warps
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t p = __shfl_up_sync(0xffffffffu, before_pages, o), q = __shfl_up_sync(0xffffffffu, before_rows, o);
        if (lane >= o) before_pages += p, before_rows += q;
    }
    if (lane == 31) warp_pages[warp] = before_pages, warp_rows[warp] = before_rows;
    __syncthreads();                                         // also: every length has been read before one is written
    int64_t all_pages = 0, all_rows = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) {
        if (w == warp) before_pages += all_pages, before_rows += all_rows;
        all_pages += warp_pages[w];
        all_rows += warp_rows[w];
    }
    before_pages -= pages;
    before_rows -= rows;
    for (int r = r0; r < r1; ++r) {
        const int need = base[r], add = starts[r];
        base[r] = (int)before_pages;
        starts[r] = (int)min(before_rows, (int64_t)a.rows);
        if (a.rows_too && blockIdx.x == 0) a.starts[r] = starts[r];
        if (a.state_too && blockIdx.x == 0) a.lengths_out[r] = (int)min((int64_t)have[r] + add, (int64_t)a.capacity);
        before_pages += need;
        before_rows += add;
    }
    if (tid == 0) {
        starts[a.requests] = (int)min(all_rows, (int64_t)a.rows);
        if (blockIdx.x == 0 && a.rows_too) a.starts[a.requests] = starts[a.requests];
        if (blockIdx.x == 0 && a.state_too) *a.taken_out = sat32(max(taken + all_pages, (int64_t)INT32_MIN));
    }
    __syncthreads();
    if (!a.rows_too) return;

    // the position in the free list of page `column` of request r, whose first new page is `first`
    const auto given = [&](int r, int column, int first) {
        const int64_t at = taken + base[r] + (column - first);
        return at >= 0 && at < a.n_free ? a.free_pages[at] : -1;
    };
    for (int64_t i = (int64_t)blockIdx.x * kPlanThreads + tid; i < all_pages; i += (int64_t)gridDim.x * kPlanThreads) {
        int low = 0, high = a.requests - 1;                  // the last request with base <= i: the one that needs page i
        while (low < high) {
            const int mid = (low + high + 1) / 2;
            if (base[mid] <= i) low = mid;
            else high = mid - 1;
        }
        const int first = (int)a.page.of(have[low] + a.page_size - 1), column = first + (int)(i - base[low]);
        a.table[low * a.ld_table + column] = given(low, column, first);
    }
    const int64_t row0 = ((int64_t)blockIdx.x * kPlanThreads + tid) * kPlanRows;
    if (row0 >= a.rows) return;
    const int live = starts[a.requests];
    int low = 0, high = a.requests;                          // the first request whose rows end behind row0, or requests
    while (low < high) {
        const int mid = (low + high) / 2;
        if (starts[mid + 1] > row0) high = mid;
        else low = mid + 1;
    }
    int64_t place[kPlanRows];
    int position[kPlanRows], number[kPlanRows];
    const int32_t* from[kPlanRows];                          // where a row's page stands
#pragma unroll
    for (int i = 0; i < kPlanRows; ++i) {
        const int64_t row = row0 + i;
        from[i] = nullptr;
        place[i] = position[i] = 0;
        if (row >= live) continue;
        while (starts[low + 1] <= row) ++low;                // row < live: there is one
        const int64_t p = have[low] + (row - starts[low]);
        position[i] = sat32(p);
        if (p >= a.capacity) continue;
        const int column = (int)a.page.of((uint32_t)p), first = (int)a.page.of(have[low] + a.page_size - 1);
        const int64_t at = taken + base[low] + (column - first);
        place[i] = p - (int64_t)column * a.page_size;
        if (column < first) from[i] = a.table + low * a.ld_table + column;
        else if (at >= 0 && at < a.n_free) from[i] = a.free_pages + at;
    }
#pragma unroll
    for (int i = 0; i < kPlanRows; ++i) number[i] = from[i] ? *from[i] : -1;
    int64_t slot[kPlanRows];
#pragma unroll
    for (int i = 0; i < kPlanRows; ++i) slot[i] = number[i] >= 0 ? (int64_t)number[i] * a.page_size + place[i] : -1;
    if (kPlanRows == 4 && a.wide && row0 + kPlanRows <= a.rows) {
        longlong2* s = reinterpret_cast<longlong2*>(a.slots + row0);
        s[0] = make_longlong2(slot[0], slot[kPlanRows / 4]);
        s[1] = make_longlong2(slot[kPlanRows / 2], slot[kPlanRows - 1]);
        *reinterpret_cast<int4*>(a.positions + row0) = make_int4(position[0], position[kPlanRows / 4], position[kPlanRows / 2], position[kPlanRows - 1]);
    } else {
#pragma unroll
        for (int i = 0; i < kPlanRows; ++i)
            if (row0 + i < a.rows) {
                a.slots[row0 + i] = slot[i];
                a.positions[row0 + i] = position[i];
            }
    }
}

// ------------------------------------------------------------------------------------------------------ append
constexpr int kAppendThreads = 256, kMaxTokens = 8, kMaxRows = 256, kAppendCtas = 4;   // the last: of an SM

struct AppendArgs {
    const void *q, *k, *v;
    void *q_out, *ck, *cv;
    float *ks, *vs;
    const int64_t* slots;
    const int32_t* positions;
    const float* inv_freq;
    int64_t q_token, q_head, o_token, o_head, k_token, k_head, v_token, v_head;
    int64_t ck_page, ck_token, ck_head, cv_page, cv_token, cv_head, n_slots;
    int heads, kv_heads, dim, page_size, pairs, interleaved, code_type, tokens, lanes, per_cta, per_part;   // the last three: VEC
};

// Cosine and sine of position * inv_freq: the angle in turns, less whole ones, in 64 bits (1 / (2 pi) as a sum of two doubles).
__device__ __forceinline__ float2 turn(int position, float inv_freq) {
    const double a = (double)position * (double)inv_freq;
    const double whole = rint(a * 0.15915494309189535), part = fma(a, -9.839338337591243e-18, fma(a, 0.15915494309189535, -whole));
    float s, c;
    sincospif(2.0f * (float)part, &s, &c);
    return make_float2(c, s);
}

__device__ __forceinline__ float max_or_nan(float a, float b) {
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}

// The scale of a row whose largest magnitude is `most` (NaN and infinity: NaN).
__device__ __forceinline__ float scale_of(float most, bool e4m3) {
    return most < INFINITY ? __fdiv_rn(most, e4m3 ? 448.0f : 127.0f) : __int_as_float(0x7fffffff);
}
// What is rounded to a code: the quotient value / scale, rounded to a float, since the product with a rounded 1 / scale (y) puts values at the
// border of two codes on the wrong side.  That product q is within two units of its last place; one step q + (x - q scale) y leaves
// 2^-22 of a unit (the remainder's and y's roundings), and is exact where the quotient is a border.  A rounded quotient that is a border, or
// next to one, could differ only for scales a few units from a fraction of few bits; at none of them does it (tests/test_code_borders.py).
// Scales below 2^-60 are brought nearer first, with their values, so that remainders stay above the smallest numbers; a scale of 0 has
// codes of 0.  16384 tokens of 16 + 2 x 16 heads of 128 to e4m3: 69.9 us; without the step 66.1, with divisions 89.5.
struct Quotient {
    float scale, up, y;
    __device__ __forceinline__ explicit Quotient(float s) : up(s < 0x1p-60f ? 0x1p64f : 1.0f) {
        scale = s * up;
        y = s == 0.0f ? 0.0f : __frcp_rn(scale);
    }
    __device__ __forceinline__ float of(float x) const {
        x *= up;
        const float q = x * y;
        return fmaf(fmaf(-q, scale, x), y, q);
    }
};

// Page and place of a slot; slots above 32 bits are rare, and their division slow.
__device__ __forceinline__ void split_slot(int64_t slot, int page_size, int64_t& page, int64_t& place) {
    if (slot >> 32) page = slot / page_size;
    else page = (uint32_t)slot / (uint32_t)page_size;
    place = slot - page * page_size;
}

// The heads of a token in one order: those of q, of k, of v.
struct Row { int kind, head; };
__device__ __forceinline__ Row row_of(const AppendArgs& a, int i) {
    if (i < a.heads) return {0, i};
    if (i < a.heads + a.kv_heads) return {1, i - a.heads};
    return {2, i - a.heads - a.kv_heads};
}

// W elements as they lie in memory, in words: copies of 16-bit element types go one by one.
template <typename T, int W> struct alignas(sizeof(T) * W > 16 ? 16 : sizeof(T) * W) Run { uint32_t word[W * sizeof(T) / 4]; };
template <int W> __device__ __forceinline__ void unpack(float (&x)[W], const Run<float, W>& r) {
#pragma unroll
    for (int i = 0; i < W; ++i) x[i] = __uint_as_float(r.word[i]);
}
template <int W> __device__ __forceinline__ void unpack(float (&x)[W], const Run<__half, W>& r) {
#pragma unroll
    for (int i = 0; i < W / 2; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&r.word[i]));
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
    }
}
template <int W> __device__ __forceinline__ void unpack(float (&x)[W], const Run<__nv_bfloat16, W>& r) {
#pragma unroll
    for (int i = 0; i < W / 2; ++i) {                        // a bf16 number is the upper half of its float
        x[2 * i] = __uint_as_float(r.word[i] << 16);
        x[2 * i + 1] = __uint_as_float(r.word[i] & 0xffff0000u);
    }
}
template <typename T, int W> __device__ __forceinline__ void store_run(T* to, const float (&x)[W]) {
    Run<T, W> r;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < W; ++i) r.word[i] = __float_as_uint(x[i]);
    } else {
#pragma unroll
        for (int i = 0; i < W / 2; ++i) {
            if constexpr (std::is_same_v<T, __half>) {
                const __half2 v = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
                r.word[i] = *reinterpret_cast<const uint32_t*>(&v);
            } else {
                const __nv_bfloat162 v = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
                r.word[i] = *reinterpret_cast<const uint32_t*>(&v);
            }
        }
    }
    *reinterpret_cast<Run<T, W>*>(to) = r;
}

// VEC: a lane has two runs of W elements of each head, the two halves of W pairs (or 2 W neighbours), so that a pair never leaves its
// lane and both its elements take the same sine; a.lanes lanes make a head.  A CTA has a.per_cta tokens and a.per_part of their heads:
// where these lie, and the turns, are worked out once and stand in shared memory, since a row itself is only some 50 instructions.
// The next row is on its way while one is worked on; four CTAs to an SM are more than a second row ahead is worth (16384 tokens of
// 64 + 2 x 8 heads of 128: 108 us, 6.2 TB/s; three CTAs and two rows ahead 118; addresses made row by row 167).  Q8: the cache holds 8 bits.
template <typename T, bool Q8, int W>
__global__ void __launch_bounds__(kAppendThreads, kAppendCtas) append_kernel(const __grid_constant__ AppendArgs a) {
    struct From { const char* src; char* dst; };             // of a head, to which a token's distance is added, in bytes
    struct By { int64_t src, dst; };
    __shared__ From head_at[kMaxRows];
    __shared__ By token_at[kMaxTokens][3];                   // of q, k and v
    __shared__ int64_t slots[kMaxTokens];                    // -1: not to be stored
    __shared__ __align__(16) float cosines[kMaxTokens][kMaxHeadDim / 2], sines[kMaxTokens][kMaxHeadDim / 2];
    constexpr int kEl = (int)sizeof(T), kCached = Q8 ? 1 : kEl;
    const int tid = threadIdx.x, lanes = a.lanes, j = tid & (lanes - 1), groups = kAppendThreads / lanes;
    const int64_t token0 = (int64_t)blockIdx.x * a.per_cta;
    const int tokens = (int)min((int64_t)a.per_cta, a.tokens - token0);
    const int row0 = blockIdx.y * a.per_part, rows = min(a.per_part, a.heads + 2 * a.kv_heads - row0);
    const int q_rows = a.heads - row0, k_rows = q_rows + a.kv_heads;         // rows below are of q, of k; the others of v
    // the runs of this lane: whole runs turn (halves), or the pairs below a.pairs (neighbours)
    const bool halves = !a.interleaved && j * W < a.pairs;
    const int run0 = halves ? j * W : 2 * j * W, run1 = halves ? a.pairs + j * W : run0 + W;
    const bool has0 = run0 < a.dim, has1 = run1 < a.dim;
    const int turned = min(max(a.pairs - j * W, 0), W);      // pairs of this lane that turn
    for (int i = tid; i < rows; i += kAppendThreads) {
        const bool is_q = i < q_rows, is_k = i < k_rows;
        const int64_t head = i - (is_q ? -row0 : is_k ? q_rows : k_rows);
        head_at[i].src = static_cast<const char*>(is_q ? a.q : is_k ? a.k : a.v) + head * (is_q ? a.q_head : is_k ? a.k_head : a.v_head) * kEl;
        head_at[i].dst = static_cast<char*>(is_q ? a.q_out : is_k ? a.ck : a.cv) + head * (is_q ? a.o_head * kEl : (is_k ? a.ck_head : a.cv_head) * kCached);
    }
    if (tid < tokens) {
        const int64_t token = token0 + tid;
        token_at[tid][0].src = token * a.q_token * kEl;
        token_at[tid][1].src = token * a.k_token * kEl;
        token_at[tid][2].src = token * a.v_token * kEl;
    }
    pdl_release();
    __syncthreads();
    pdl_wait();

    struct Item { int t, row; };                             // rows of a token, then of the next, `groups` apart
    const auto settle = [&](Item& i) {
        while (i.row >= rows && i.t < tokens) i.row -= rows, ++i.t;
    };
    Run<T, W> raw[2] = {};                                   // the next row's runs, zeros where nothing is read
    Item asked{0, tid / lanes};
    settle(asked);
    const auto fetch = [&] {
        if (asked.t < tokens) {
            const char* p = head_at[asked.row].src + token_at[asked.t][asked.row < q_rows ? 0 : asked.row < k_rows ? 1 : 2].src;
            if (has0) raw[0] = *reinterpret_cast<const Run<T, W>*>(p + run0 * kEl);
            if (has1) raw[1] = *reinterpret_cast<const Run<T, W>*>(p + run1 * kEl);
        }
        asked.row += groups;
        settle(asked);
    };
    fetch();
    // under the first rows' way: where the tokens go, and the turns
    if (tid < tokens) {
        const int64_t token = token0 + tid, slot = a.slots[token];
        const bool stored = slot >= 0 && slot < a.n_slots;
        int64_t page = 0, place = 0;
        if (stored) split_slot(slot, a.page_size, page, place);
        slots[tid] = stored ? slot : -1;
        token_at[tid][0].dst = token * a.o_token * kEl;
        token_at[tid][1].dst = (page * a.ck_page + place * a.ck_token) * kCached;
        token_at[tid][2].dst = (page * a.cv_page + place * a.cv_token) * kCached;
    }
    for (int i = tid; i < tokens * a.pairs; i += kAppendThreads) {
        const int t = i / a.pairs, pair = i - t * a.pairs;
        const float2 by = turn(a.positions[token0 + t], a.inv_freq[pair]);
        cosines[t][pair] = by.x;
        sines[t][pair] = by.y;
    }
    __syncthreads();
    Item at{0, tid / lanes};
    settle(at);
    const int loops = (tokens * rows + groups - 1) / groups; // the same for every thread: shuffles need them all
#pragma unroll 1
    for (int n = 0; n < loops; ++n) {
        const bool live = at.t < tokens;
        const int t = live ? at.t : 0, row = live ? at.row : 0, kind = row < q_rows ? 0 : row < k_rows ? 1 : 2;
        float x[W], y[W];
        unpack(x, raw[0]);
        unpack(y, raw[1]);
        fetch();
        if (turned && kind < 2) {
            float cosine[W], sine[W];
#pragma unroll
            for (int e = 0; e < W; e += 4) {
                *reinterpret_cast<float4*>(cosine + e) = *reinterpret_cast<const float4*>(&cosines[t][j * W + e]);
                *reinterpret_cast<float4*>(sine + e) = *reinterpret_cast<const float4*>(&sines[t][j * W + e]);
            }
            if (!a.interleaved) {
#pragma unroll
                for (int e = 0; e < W; ++e) {
                    const float u = x[e];
                    x[e] = fmaf(u, cosine[e], -y[e] * sine[e]);
                    y[e] = fmaf(u, sine[e], y[e] * cosine[e]);
                }
            } else {                                         // element 2 e of the 2 W neighbours and the one behind it
#pragma unroll
                for (int e = 0; e < W; ++e) {
                    float &p = e < W / 2 ? x[2 * (e % (W / 2))] : y[2 * (e % (W / 2))], &q = e < W / 2 ? x[2 * (e % (W / 2)) + 1] : y[2 * (e % (W / 2)) + 1];
                    const float u = p;
                    if (e < turned) {
                        p = fmaf(u, cosine[e], -q * sine[e]);
                        q = fmaf(u, sine[e], q * cosine[e]);
                    }
                }
            }
        }
        char* to = head_at[row].dst + token_at[t][kind].dst;
        if (!Q8 || kind == 0) {
            if (live && (kind == 0 || slots[t] >= 0)) {
                if (has0) store_run(reinterpret_cast<T*>(to) + run0, x);
                if (has1) store_run(reinterpret_cast<T*>(to) + run1, y);
            }
        }
        if (Q8 && __any_sync(0xffffffffu, kind != 0 && live)) {
            const bool e4m3 = a.code_type == PP_E4M3;
            float most = 0.0f;
#pragma unroll
            for (int e = 0; e < W; ++e) most = max_or_nan(max_or_nan(most, fabsf(x[e])), fabsf(y[e]));
            for (int o = 1; o < lanes; o <<= 1) most = max_or_nan(most, __shfl_xor_sync(0xffffffffu, most, o));
            if (kind != 0 && live && slots[t] >= 0) {
                const float scale = scale_of(most, e4m3);
                Run<uint8_t, W> u, w;
                const Quotient over(scale);
#pragma unroll
                for (int e = 0; e < W; ++e) x[e] = over.of(x[e]), y[e] = over.of(y[e]);
#pragma unroll
                for (int e = 0; e < W; e += 4) u.word[e / 4] = four_codes(x + e, e4m3), w.word[e / 4] = four_codes(y + e, e4m3);
                if (has0) *reinterpret_cast<Run<uint8_t, W>*>(to + run0) = u;
                if (has1) *reinterpret_cast<Run<uint8_t, W>*>(to + run1) = w;
                if (j == 0) (kind == 1 ? a.ks : a.vs)[slots[t] * a.kv_heads + (row - (kind == 1 ? q_rows : k_rows))] = scale;
            }
        }
        at.row += groups;
        settle(at);
    }
}

// Any width and alignment: a warp to a head, element by element.
template <typename T>
__global__ void __launch_bounds__(kAppendThreads) append_any_kernel(const AppendArgs a) {
    constexpr int kPer = kMaxHeadDim / 32;
    __shared__ float2 turns[kMaxHeadDim / 2];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t token = blockIdx.x;
    const int rows = a.heads + 2 * a.kv_heads;
    pdl_release();
    pdl_wait();
    const int64_t slot = a.slots[token];
    if (a.pairs) {
        const int position = a.positions[token];
        for (int i = tid; i < a.pairs; i += kAppendThreads) turns[i] = turn(position, a.inv_freq[i]);
        __syncthreads();
    }
    const bool stored = slot >= 0 && slot < a.n_slots;
    int64_t page = 0, place = 0;
    if (stored) split_slot(slot, a.page_size, page, place);
    for (int i = blockIdx.y * (kAppendThreads / 32) + warp; i < rows; i += gridDim.y * (kAppendThreads / 32)) {
        const Row r = row_of(a, i);
        const T* src = r.kind == 0 ? static_cast<const T*>(a.q) + token * a.q_token + r.head * a.q_head
                     : r.kind == 1 ? static_cast<const T*>(a.k) + token * a.k_token + r.head * a.k_head
                                   : static_cast<const T*>(a.v) + token * a.v_token + r.head * a.v_head;
        float x[kPer];
        float most = 0.0f;
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const int d = lane + 32 * e;
            x[e] = 0.0f;
            if (d >= a.dim) continue;
            x[e] = to_float(src[d]);
            if (r.kind < 2 && d < 2 * a.pairs) {
                const bool second = a.interleaved ? (d & 1) : d >= a.pairs;
                const float2 t = turns[a.interleaved ? d / 2 : second ? d - a.pairs : d];
                const float y = to_float(src[a.interleaved ? d ^ 1 : second ? d - a.pairs : d + a.pairs]);
                x[e] = fmaf(x[e], t.x, y * (second ? t.y : -t.y));
            }
            most = max_or_nan(most, fabsf(x[e]));
        }
        __syncwarp();                                        // q_out may be q: every lane has read what another will write
        if (r.kind == 0) {
            T* dst = static_cast<T*>(a.q_out) + token * a.o_token + r.head * a.o_head;
#pragma unroll
            for (int e = 0; e < kPer; ++e)
                if (lane + 32 * e < a.dim) dst[lane + 32 * e] = from_float<T>(x[e]);
            continue;
        }
        if (!stored) continue;
        const int64_t at = r.kind == 1 ? page * a.ck_page + place * a.ck_token + r.head * a.ck_head : page * a.cv_page + place * a.cv_token + r.head * a.cv_head;
        void* cache = r.kind == 1 ? a.ck : a.cv;
        if (a.code_type == PP_E4M3 || a.code_type == PP_I8) {
            const bool e4m3 = a.code_type == PP_E4M3;
#pragma unroll
            for (int o = 16; o; o >>= 1) most = max_or_nan(most, __shfl_xor_sync(0xffffffffu, most, o));
            const float scale = scale_of(most, e4m3);
            uint8_t* dst = static_cast<uint8_t*>(cache) + at;
            const Quotient over(scale);
#pragma unroll
            for (int e = 0; e < kPer; ++e) x[e] = over.of(x[e]);
#pragma unroll
            for (int e = 0; e < kPer; e += 4) {
                const uint32_t four = four_codes(x + e, e4m3);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (lane + 32 * (e + i) < a.dim) dst[lane + 32 * (e + i)] = (uint8_t)(four >> (8 * i));
            }
            if (lane == 0) (r.kind == 1 ? a.ks : a.vs)[slot * a.kv_heads + r.head] = scale;
        } else {
            T* dst = static_cast<T*>(cache) + at;
#pragma unroll
            for (int e = 0; e < kPer; ++e)
                if (lane + 32 * e < a.dim) dst[lane + 32 * e] = from_float<T>(x[e]);
        }
    }
}

template <typename T, bool Q8> cudaError_t launch_append(AppendArgs& a, int width, cudaStream_t stream) {
    if (width) {
        const int runs = (a.dim + 2 * width - 1) / (2 * width);
        a.lanes = 1;
        while (a.lanes < runs) a.lanes *= 2;
    }
    const int rows = a.heads + 2 * a.kv_heads;
    const int at_once = width ? kAppendThreads / a.lanes : kAppendThreads / 32;
    // a CTA per token where tokens fill the GPU; else a token's heads are divided, down to one to a group of lanes
    int parts = width ? (rows + kMaxRows - 1) / kMaxRows : 1;
    while (parts * at_once < rows && (int64_t)a.tokens * parts < 4 * (int64_t)sm_count()) ++parts;
    a.per_part = (rows + parts - 1) / parts;
    parts = (rows + a.per_part - 1) / a.per_part;
    // many tokens: as many to a CTA, up to eight, as leave the fewest to the CTAs that one place of an SM runs in turn, with one more for
    // each CTA's start (four to a CTA against this rule: 16384 tokens of 64 + 2 x 8 heads of 128 by seven 108.5, 107.9 us; 4095 of 16-bit
    // heads of 256 17.2, 16.5; others of thousands of tokens 43.3, 39.6 and 21.3, 17.0)
    if (width && a.tokens >= 16 * sm_count()) {
        const int64_t at_once = (int64_t)sm_count() * kAppendCtas;
        int64_t least = INT64_MAX;
        for (int per = 1; per <= kMaxTokens; ++per) {
            const int64_t cost = (((int64_t)a.tokens + per - 1) / per * parts + at_once - 1) / at_once * (per + 1);
            if (cost < least) least = cost, a.per_cta = per;
        }
    }
    const dim3 grid((unsigned)(((int64_t)a.tokens + a.per_cta - 1) / a.per_cta), (unsigned)parts);
    return launch_pdl(width == 8 ? append_kernel<T, Q8, sizeof(T) == 4 ? 4 : 8> : width == 4 ? append_kernel<T, Q8, 4> : append_any_kernel<T>, grid, dim3(kAppendThreads), 0, stream, 1, a);
}

}  // namespace
}  // namespace pp

extern "C" pp_status_t pp_paged_plan(const int32_t* lengths, const int32_t* added, int32_t* table, int64_t ld_table, int width,
                                     const int32_t* free_pages, int n_free, const int32_t* taken, int requests, int page_size, int rows,
                                     int64_t* slots, int32_t* positions, int32_t* starts, int32_t* lengths_out, int32_t* taken_out,
                                     void* cuda_stream) {
    using namespace pp;
    if (requests < 0 || width < 1 || page_size < 1 || rows < 0 || n_free < 0 || !taken || !starts || !taken_out) return PP_ERR_INVALID_ARG;
    if (requests > 0 && (!lengths || !added || !table || !lengths_out || ld_table < width)) return PP_ERR_INVALID_ARG;
    if ((rows > 0 && (!slots || !positions)) || (n_free > 0 && !free_pages)) return PP_ERR_INVALID_ARG;
    const int64_t capacity = (int64_t)width * page_size;
    // a length rounded up to pages and the pages of all requests fit 32 bits
    if (requests > kMaxRequests || capacity > INT32_MAX - page_size || (int64_t)requests * width > INT32_MAX) return PP_ERR_UNSUPPORTED;
    if (ld_table > ((int64_t)1 << 40)) return PP_ERR_INVALID_ARG;
    for (const void* p : {(const void*)lengths, (const void*)added, (const void*)table, (const void*)free_pages, (const void*)taken,
                          (const void*)positions, (const void*)starts, (const void*)lengths_out, (const void*)taken_out})
        if (!aligned_to(p, 4)) return PP_ERR_INVALID_ARG;
    if (!aligned_to(slots, 8)) return PP_ERR_INVALID_ARG;
    const int64_t n = requests;
    struct Span { const void* p; int64_t bytes; };
    const Span in[] = {{lengths, 4 * n}, {added, 4 * n}, {free_pages, 4 * (int64_t)n_free}, {taken, 4}};
    const Span out[] = {{table, n ? 4 * ((n - 1) * ld_table + width) : 0}, {slots, 8 * (int64_t)rows}, {positions, 4 * (int64_t)rows},
                        {starts, 4 * (n + 1)}, {lengths_out, 4 * n}, {taken_out, 4}};
    for (const Span& o : out) {
        for (const Span& i : in) {
            const bool in_place = o.p == i.p && ((i.p == lengths && o.p == lengths_out) || (i.p == taken && o.p == taken_out));
            if (!in_place && spans_meet(o.p, o.bytes, i.p, i.bytes)) return PP_ERR_INVALID_ARG;
        }
        for (const Span& other : out)
            if (&other != &o && spans_meet(o.p, o.bytes, other.p, other.bytes)) return PP_ERR_INVALID_ARG;
    }
    PlanArgs a{lengths, added, free_pages, taken, table, slots, positions, starts, lengths_out, taken_out, ld_table,
               width, n_free, requests, page_size, rows, (int)capacity, Divisor((uint32_t)page_size), aligned_to(slots, 16) && aligned_to(positions, 16), true, true};
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const size_t smem = (3 * (size_t)requests + 1) * 4;
    // a row to a thread while one CTA holds them, or while CTAs are few; then four
    const bool one = rows <= kPlanThreads || (rows > 4 * kPlanThreads && rows <= 2 * kPlanThreads * sm_count());
    const auto kernel = one ? plan_kernel<1> : plan_kernel<4>;
    static PerDeviceOnce opt_in[2];
    int device = 0;
    if (const cudaError_t e = cudaGetDevice(&device)) return status_of(e);
    // 48 KB that a launch has by itself are for the kernel's own arrays too: asked for well below
    if (smem > 32 * 1024 && !opt_in[one].is_done(device)) {
        if (const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (3 * kMaxRequests + 1) * 4)) return status_of(e);
        opt_in[one].mark(device);
    }
    const int64_t per = kPlanThreads * (one ? 1 : 4);
    const unsigned grid = (unsigned)std::max<int64_t>(1, (rows + per - 1) / per);
    // In place and with several CTAs, one would write a length that another has still to read: lengths and pages taken are then
    // written by a launch of their own, behind the first.
    const bool apart = grid > 1 && (lengths == lengths_out || taken == taken_out);
    a.state_too = !apart;
    cudaError_t e = launch_pdl(kernel, dim3(grid), dim3(kPlanThreads), smem, stream, 1, a);
    if (e == cudaSuccess && apart) {
        a.rows_too = false;
        a.state_too = true;
        e = launch_pdl(kernel, dim3(1), dim3(kPlanThreads), smem, stream, 1, a);
    }
    return status_of(e);
}

extern "C" pp_status_t pp_kv_append(const pp_paged_cache_t* cache, const void* q, int64_t q_token, int64_t q_head, int heads, void* q_out,
                                    int64_t o_token, int64_t o_head, const void* k, int64_t k_token, int64_t k_head, const void* v,
                                    int64_t v_token, int64_t v_head, pp_dtype_t dtype, int tokens, const int64_t* slots,
                                    const int32_t* positions, const float* inv_freq, int pairs, int interleaved, void* cuda_stream) {
    using namespace pp;
    if (const pp_status_t st = check_cache(cache)) return st;
    const pp_paged_cache_t& c = *cache;
    if (!is_float(dtype) || (c.dtype != dtype && !is_8bit(c.dtype))) return PP_ERR_UNSUPPORTED;
    if (tokens < 0 || heads < 0 || heads > (1 << 20) || pairs < 0 || pairs > c.head_dim / 2 || (heads > 0) != (q != nullptr) || (q != nullptr) != (q_out != nullptr))
        return PP_ERR_INVALID_ARG;
    if ((pairs > 0) != (positions != nullptr) || (pairs > 0) != (inv_freq != nullptr)) return PP_ERR_INVALID_ARG;
    if (tokens == 0) return PP_OK;
    if (!k || !v || !slots) return PP_ERR_INVALID_ARG;
    const int tb = type_bytes(dtype), dim = c.head_dim;
    if (!aligned_to(q, tb) || !aligned_to(q_out, tb) || !aligned_to(k, tb) || !aligned_to(v, tb) || !aligned_to(slots, 8) || !aligned_to(positions, 4) ||
        !aligned_to(inv_freq, 4)) return PP_ERR_INVALID_ARG;
    const int64_t most = (int64_t)1 << 58;                   // no sum of offsets passes 63 bits
    for (const int64_t s : {q_token, o_token, k_token, v_token})
        if (s < 0 || s > most / tokens) return PP_ERR_INVALID_ARG;
    for (const int64_t s : {q_head, o_head, k_head, v_head})
        if (s < 0 || s > most >> 20) return PP_ERR_INVALID_ARG;
    const Held held(c);
    if (held.meet(slots, 8 * (int64_t)tokens) || held.meet(positions, 4 * (int64_t)tokens) || held.meet(inv_freq, 4 * (int64_t)pairs))
        return PP_ERR_INVALID_ARG;
    const auto span = [&](int64_t token, int64_t head, int n) { return (((int64_t)tokens - 1) * token + ((int64_t)n - 1) * head + dim) * tb; };
    if (q) {
        if (!rows_apart(1, 0, tokens, o_token, heads, o_head, dim)) return PP_ERR_INVALID_ARG;
        const bool in_place = q == q_out && q_token == o_token && q_head == o_head;
        // A token's rows of each array, q_token (k_token ...) apart: arrays with one distance may lie in one another's gaps, as the parts of a
        // projection's rows do; others may not meet at all.
        const int64_t out_row = (((int64_t)heads - 1) * o_head + dim) * tb;
        const auto meets = [&](const void* p, int64_t token, int64_t head, int n) {
            const int64_t row = (((int64_t)n - 1) * head + dim) * tb;
            if (token == o_token) return share_bytes(q_out, out_row, o_token * tb, tokens, p, row, token * tb, tokens);
            return spans_meet(p, span(token, head, n), q_out, span(o_token, o_head, heads));
        };
        // the cache is written too, and what says where to is read meanwhile
        const Rows turned(q_out, 1, 0, tokens, o_token, heads, o_head, dim, tb);
        if (held.meet(q_out, turned.span()) || turned.meet(slots, 8 * (int64_t)tokens) || turned.meet(positions, 4 * (int64_t)tokens) ||
            turned.meet(inv_freq, 4 * (int64_t)pairs)) return PP_ERR_INVALID_ARG;
        if ((!in_place && meets(q, q_token, q_head, heads)) || meets(k, k_token, k_head, c.kv_heads) || meets(v, v_token, v_head, c.kv_heads)) return PP_ERR_INVALID_ARG;
    }
    AppendArgs a{q, k, v, q_out, c.k, c.v, c.k_scales, c.v_scales, slots, positions, inv_freq,
                 q_token, q_head, o_token, o_head, k_token, k_head, v_token, v_head,
                 c.k_page, c.k_token, c.k_head, c.v_page, c.v_token, c.v_head, (int64_t)c.pages * c.page_size,
                 heads, c.kv_heads, dim, c.page_size, pairs, interleaved != 0, c.dtype, tokens, 1, 1, 1};
    // eight or four elements to an access where every row starts on one, and runs of pairs are whole ones
    const auto alignment = [&](const void* p, int64_t token, int64_t head, int n) { return !p ? 16 : row_alignment(p, 1, 0, tokens, token, n, head, tb); };
    const int rows_on = std::min({alignment(q, q_token, q_head, heads), alignment(q_out, o_token, o_head, heads), alignment(k, k_token, k_head, c.kv_heads),
                                  alignment(v, v_token, v_head, c.kv_heads)}), cache_on = cache_alignment(c);
    const auto fits = [&](int w) {
        return dim % w == 0 && (interleaved || pairs % w == 0) && rows_on >= std::min(16, w * tb) && cache_on >= std::min(16, w * type_bytes(c.dtype));
    };
    const int width = dtype != PP_F32 && fits(8) ? 8 : fits(4) ? 4 : 0;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    const bool q8 = is_8bit(c.dtype);
    const cudaError_t e = dtype == PP_F32   ? (q8 ? launch_append<float, true>(a, width, s) : launch_append<float, false>(a, width, s))
                          : dtype == PP_F16 ? (q8 ? launch_append<__half, true>(a, width, s) : launch_append<__half, false>(a, width, s))
                                            : (q8 ? launch_append<__nv_bfloat16, true>(a, width, s) : launch_append<__nv_bfloat16, false>(a, width, s));
    return status_of(e);
}
