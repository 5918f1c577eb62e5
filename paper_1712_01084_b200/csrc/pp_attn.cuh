// Attention of one new token of each request over a paged key-value cache: the kernels (pp_attn.cu has the choice among them).
//
//   out = sum_j p_j v_j,  p = softmax_j(scale q . k_j),  j over a request's last positions
//
// One pass over keys and values with a running maximum m and sum l: bound by the bytes of the cache, which are read once for a chunk of
// query heads of a key-value head, 16 of them up to 128 dimensions and 8 above, in floats, and for float q over 8 bits.  Chunks of one
// head are heads of their own in what follows: more query heads than a chunk read the cache again, from L2 while it holds it.  m only
// moves when a score passes it by 2^8: then sums and l are scaled; else a tile costs one vote.
//
// Division of work.  64 positions of one key-value head (and chunk) are a unit, 16 to a warp; or 16 positions of four heads, one
// to a warp, where the heads' rows or scales share lines of memory.  Three ways (divide in pp_attn.cu):
//   * equal parts: the units of all requests in a row, request after request and head after head, are cut into equal parts, one
//     for each CTA that the GPU holds at once, so that lengths of any mix keep all SMs reading to the end.  A CTA finds its part
//     from the lengths alone.  Where a cut falls inside a head's units the CTAs write partial results (m, l, the weighted sum)
//     to the workspace, and a second kernel joins them in the order of the sequence;
//   * a cluster of two to eight CTAs to a head: each sends its part of a row to the CTA that joins it, over shared memory;
//   * a CTA to a head, or to four.
//
// A warp takes tiles of 16 positions of its own, through a ring in shared memory that 16-byte asynchronous copies fill.  Pages may
// have any size and end anywhere; where they are whole tiles long a tile costs one look-up, its entries fetched 32 tiles at a
// time, else every row has its own.  Rows are an odd number of 16 bytes apart, so that eight of them meet no bank twice.
//
// Matrix form (MmaCore), S^T[16 positions x 8 heads] = K Q^T and O^T[dim x 8 heads] += V^T P^T, by m16n8k16: the cache is the operand
// with 16 rows, heads are the eight columns, so no instruction works on padding where a key-value head has eight query heads.
// Not tcgen05: with 8 to 16 heads to a row of the cache the matrix pipe is busy 15 to 19 % of the time, and codes have to pass
// through registers to be widened.  P^T changes from the layout of a result to that of an operand by 8x8 transposes in registers;
// it enters as two 16-bit numbers, the rounded value and what the rounding left (one alone would add an error as large as the
// output's own rounding), or as one where that is an eighth of it.  8-bit codes are exact in f16; the scale of a key multiplies
// its score, that of a value its p.
// Scalar form (ScalarCore): floats, a lane per position and half row for the scores, a lane per dimension for the sums.
//
// In a graph, heads of 128, 32 query heads over 8: 64 requests of 4096 to 8192 bf16 247 to 252 us, 6.5 TB/s of what they hold; one of
// 131072 91 to 93 us, 5.8 TB/s; 33 of 6000 to 12000 in 8 bits with 64 heads 120 to 123 us, 5.2 TB/s; one of 513 6.4 us; 6 of 500 to 1000
// floats, 16 heads of 64, 12.0 us.
#pragma once
#include "pp_internal.h"
#include "pp_paged.cuh"

namespace pp {
namespace attn {


constexpr int kWarps = 4, kThreads = kWarps * 32, kTile = 16, kUnit = kWarps * kTile;
constexpr int kAheadMost = 8192;
static_assert(kAheadMost > 65 * kUnit);
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

struct AttnArgs {
    const void* q;
    const char *k, *v;                                       // strides below in bytes
    const float *ks, *vs;
    const int32_t *table, *lengths;
    void* out;
    float *lse, *ws;
    int64_t q_row, q_head, k_page, k_token, k_head, v_page, v_token, v_head, ld_table;
    Divisor page;
    int pages, page_size, batch, capacity, window, heads, kv_heads, group, chunk, n_chunks, dim, granule, q_type, type;
    int inbox;                                               // where a cluster's CTAs write in each other's shared memory, in bytes
    int notes, part_rows;                                    // in the workspace; rows of a partial result
    bool by_head;                                            // a note's place is the head's, not the CTA's
    int cluster;                                             // CTAs that share a head (chunk); 0: all heads in a row, cut into equal parts
    // A unit of work: 64 positions of one key-value head, 16 to a warp, or (across) 16 positions of four heads, one to a warp
    int unit, unit_in_page;                                  // its positions; these modulo the page size
    bool across;
    bool whole_tiles;                                        // no tile crosses pages, distances fit 32 bits, and pieces are 16 or 8 bytes
    bool wide_out;                                           // four neighbours of out are one access
    float scale;                                             // times log2 e
};

// The workspace: a note for each CTA (four ints), then two partial results for each.  A partial result: m and l of each row,
// then their sums, all on 16 bytes.
__host__ __device__ inline int64_t notes_floats(int64_t ctas) { return 4 * ctas; }
__host__ __device__ inline int up4(int n) { return (n + 3) & ~3; }
__host__ __device__ inline int64_t part_floats(int rows, int dim) { return 2 * up4(rows) + (int64_t)rows * up4(dim); }

__device__ __forceinline__ int first_position(const AttnArgs& a, int length) { return a.window > 0 ? max(0, length - a.window) : 0; }
// Units start at a whole tile: where pages are whole tiles long, no tile then crosses from one page into another.
__device__ __forceinline__ int first_tile(const AttnArgs& a, int length) { return first_position(a, length) & ~(kTile - 1); }
__device__ __forceinline__ int length_of(const AttnArgs& a, int r) { return min(max(a.lengths[r], 0), a.capacity); }
// Units of one head of a request: one at least, which writes the output of a request without positions.
__device__ __forceinline__ int units_of(const AttnArgs& a, int r) {
    const int n = length_of(a, r);
    return max(1, (n - first_tile(a, n) + a.unit - 1) / a.unit);
}

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t smem_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

// The q rows of a chunk as floats [heads][DT] in shared memory, zeros where there is no head or dimension.
template <int HEADS, int DT, typename T> __device__ __forceinline__ void stage_q(const AttnArgs& a, const T* q, int n_heads, float* to) {
#pragma unroll 8
    for (int i = threadIdx.x; i < HEADS * DT; i += kThreads) {
        const int head = i / DT, d = i - head * DT;
        to[i] = head < n_heads && d < a.dim ? to_float(q[head * a.q_head + d]) : 0.0f;
    }
}
template <int HEADS, int DT> __device__ __forceinline__ void stage_q(const AttnArgs& a, int r, int head0, int n_heads, float* to) {
    const int64_t at = r * a.q_row + head0 * a.q_head;
    if (a.q_type == PP_BF16) stage_q<HEADS, DT>(a, static_cast<const __nv_bfloat16*>(a.q) + at, n_heads, to);
    else if (a.q_type == PP_F16) stage_q<HEADS, DT>(a, static_cast<const __half*>(a.q) + at, n_heads, to);
    else stage_q<HEADS, DT>(a, static_cast<const float*>(a.q) + at, n_heads, to);
}
// Dimensions d .. d + 3 of a row of out.
__device__ __forceinline__ void store_out(const AttnArgs& a, int64_t row, int d, float4 v) {
    const int64_t at = row * a.dim + d;
    if (a.wide_out) {
        if (a.q_type == PP_F32) {
            *reinterpret_cast<float4*>(static_cast<float*>(a.out) + at) = v;
        } else if (a.q_type == PP_F16) {
            const __half2 x = __floats2half2_rn(v.x, v.y), y = __floats2half2_rn(v.z, v.w);
            *reinterpret_cast<uint2*>(static_cast<__half*>(a.out) + at) = make_uint2(*reinterpret_cast<const uint32_t*>(&x), *reinterpret_cast<const uint32_t*>(&y));
        } else {
            const __nv_bfloat162 x = __floats2bfloat162_rn(v.x, v.y), y = __floats2bfloat162_rn(v.z, v.w);
            *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.out) + at) = make_uint2(*reinterpret_cast<const uint32_t*>(&x), *reinterpret_cast<const uint32_t*>(&y));
        }
        return;
    }
    const float f[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (d + i >= a.dim) break;
        if (a.q_type == PP_F32) static_cast<float*>(a.out)[at + i] = f[i];
        else if (a.q_type == PP_F16) static_cast<__half*>(a.out)[at + i] = __float2half_rn(f[i]);
        else static_cast<__nv_bfloat16*>(a.out)[at + i] = __float2bfloat16_rn(f[i]);
    }
}
__device__ __forceinline__ float4 add4(float4 a, float4 b) { return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w); }
__device__ __forceinline__ float4 fma4(float4 a, float by, float4 b) { return make_float4(fmaf(a.x, by, b.x), fmaf(a.y, by, b.y), fmaf(a.z, by, b.z), fmaf(a.w, by, b.w)); }
// A sum over l, 0 where nothing was summed.
__device__ __forceinline__ float4 over(float4 v, float l) {
    if (l == 0.0f) return make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    return make_float4(__fdiv_rn(v.x, l), __fdiv_rn(v.y, l), __fdiv_rn(v.z, l), __fdiv_rn(v.w, l));
}
// A running maximum starts at the lowest float, not at minus infinity: no difference of two of them is then a NaN.  It need not be the
// maximum: it moves when a score is more than 2^kSlack above it, so that most tiles pass with one vote and no exchange of maxima.
constexpr float kLowest = -3.402823466e38f, kSlack = 8.0f;
__device__ __forceinline__ float weight_of(float m, float top) { return exp2_fast(m - top); }
// 2^n for n < 128, 0 below the normal numbers; and the power of two of a positive number (-127 for what is smaller than normal ones).
__device__ __forceinline__ float power(int n) { return n < -126 ? 0.0f : __int_as_float((n + 127) << 23); }
__device__ __forceinline__ int exponent(float x) { return ((__float_as_int(x) >> 23) & 255) - 127; }

template <int BYTES> __device__ __forceinline__ void copy_async(uint32_t dst, const void* src, bool there) {   // zeros if not there
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(BYTES), "r"(there ? BYTES : 0) : "memory");
}
__device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void wait_but() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// How a kernel reads: whole tiles in pieces of 16 bytes; whole tiles in pieces of 8 bytes, or row by row in pieces of 16, 8 or 4; element
// by element.  Kernels of their own: the look-ups of the second in the first one's way cost it up to 7 %, and called as a function
// they cost themselves 10 to 20 %.
enum Reading { kWhole, kRows, kElements };

// What a warp reads: positions of one request and key-value head, in tiles a.unit apart.
struct Reader {
    const char *k, *v;
    const float *ks, *vs;
    const int32_t* row;                                      // of the table
    int low, end;                                            // positions low .. end - 1 count
    int at, n, place;                                        // the next tile: its position, its number, and where in its page it starts
    int entry, next;                                         // table entries, see below
};

// Table entries.  In whole tiles (a.whole_tiles) lane i holds that of the i-th tile of a batch of 32, and of the batch behind it;
// otherwise that of position lane & 15 of the next tile.  -1: not asked for.
__device__ __forceinline__ int entry_of(const AttnArgs& a, const Reader& r, int at) { return at < r.end ? r.row[a.page.of((uint32_t)at)] : -1; }
__device__ __forceinline__ int position_entry(const AttnArgs& a, const Reader& r, int at) {
    const int p = at + (threadIdx.x & 15);
    return p >= r.low ? entry_of(a, r, p) : -1;
}
__device__ __forceinline__ void start(const AttnArgs& a, Reader& r) {
    r.n = 0;
    if (a.whole_tiles) {
        r.place = r.at - (int)a.page.of((uint32_t)r.at) * a.page_size;
        r.next = entry_of(a, r, r.at + (int)(threadIdx.x & 31) * a.unit);
    } else {
        r.entry = position_entry(a, r, r.at);
    }
}
// Bits of the tile's positions between low and end.
__device__ __forceinline__ uint32_t positions_of(const Reader& r, int at) {
    const int from = max(0, r.low - at), to = min(kTile, r.end - at);
    return ((1u << to) - 1u) & ~((1u << from) - 1u);
}

// Rows that are looked up one by one, in pieces of a.granule bytes.  Returns which rows are there (a bit each).
template <int ES, int CHUNKS, int PITCH, bool Q8>
__device__ __forceinline__ uint32_t ask_by_row(const AttnArgs& a, const char* k, const char* v, const float* ks, const float* vs, int low, int end, int entry, int at,
                                            uint32_t stage) {
    constexpr int kTileBytes = kTile * PITCH;
    const int lane = threadIdx.x & 31, p = at + (lane & 15);
    const bool there = p >= low && p < end && (uint32_t)entry < (uint32_t)a.pages;   // -1 is no page, and a number that is none of the cache's neither
    const uint32_t bits = __ballot_sync(0xffffffffu, there) & 0xffffu;
    int64_t off = 0;
    int place = 0;
    if (there) {
        place = p - (int)a.page.of((uint32_t)p) * a.page_size;
        off = lane < 16 ? (int64_t)entry * a.k_page + (int64_t)place * a.k_token : (int64_t)entry * a.v_page + (int64_t)place * a.v_token;
    }
    const auto copy = [&](auto bytes) {
        constexpr int B = decltype(bytes)::value, kPieces = CHUNKS * 16 / B;
        constexpr int kLanes = kPieces > 16 ? 32 : kPieces > 8 ? 16 : kPieces > 4 ? 8 : 4;
        const int own = a.dim * ES / B;
#pragma unroll 2
        for (int i = 0; i < kTile * kLanes / 32; ++i) {
            const int row = i * (32 / kLanes) + lane / kLanes;
            const int64_t ko = __shfl_sync(0xffffffffu, off, row), vo = __shfl_sync(0xffffffffu, off, 16 + row);
            const bool has = (bits >> row) & 1;
            for (int c = lane & (kLanes - 1); c < kPieces; c += kLanes) {
                const bool in = has && c < own;
                const int piece = in ? c * B : 0;
                copy_async<B>(stage + row * PITCH + c * B, k + ko + piece, in);
                copy_async<B>(stage + kTileBytes + row * PITCH + c * B, v + vo + piece, in);
            }
        }
    };
    if (a.granule == 16) copy(std::integral_constant<int, 16>());
    else if (a.granule == 8) copy(std::integral_constant<int, 8>());
    else copy(std::integral_constant<int, 4>());
    if constexpr (Q8) {
        const int64_t token = there ? (int64_t)entry * a.page_size + place : 0;
        copy_async<4>(stage + 2 * kTileBytes + lane * 4, (lane < 16 ? ks : vs) + token * a.kv_heads, there);
    }
    return bits;
}

// The same for rows a fixed distance apart, in pieces of 8 bytes.
template <int CHUNKS, int PITCH>
__device__ __forceinline__ void ask_eights(const char* k, const char* v, uint32_t k_token, uint32_t v_token, int own, uint32_t bits, uint32_t stage) {
    constexpr int kPieces = CHUNKS * 2, kLanes = kPieces > 16 ? 32 : kPieces > 8 ? 16 : 8, kRows = 32 / kLanes;
    const int lane = threadIdx.x & 31, row = lane / kLanes;
    for (int c = lane & (kLanes - 1); c < kPieces; c += kLanes) {
        const bool in = c < own;
#pragma unroll 4
        for (int i = row; i < kTile; i += kRows) {
            const bool has = in && ((bits >> i) & 1);
            copy_async<8>(stage + i * PITCH + c * 8, k + (uint64_t)i * k_token + (in ? c * 8 : 0), has);
            copy_async<8>(stage + kTile * PITCH + i * PITCH + c * 8, v + (uint64_t)i * v_token + (in ? c * 8 : 0), has);
        }
    }
}

// Asks for the next tile: 16 rows of keys, of values, and the scales of both.  Returns which rows are there.
// ES: bytes of an element, CHUNKS: 16-byte pieces of a row as the kernel sees it (rows that are shorter end in zeros).
template <int ES, int CHUNKS, int PITCH, bool Q8, Reading READING>
__device__ __forceinline__ uint32_t ask(const AttnArgs& a, Reader& r, uint32_t stage) {
    constexpr int kTileBytes = kTile * PITCH;
    constexpr int kLanes = CHUNKS > 16 ? 32 : CHUNKS > 8 ? 16 : CHUNKS > 4 ? 8 : 4, kRows = 32 / kLanes;
    const int lane = threadIdx.x & 31, at = r.at;
    r.at += a.unit;
    if (READING != kWhole && !a.whole_tiles) {
        const int found = r.entry;
        r.entry = position_entry(a, r, r.at);
        return ask_by_row<ES, CHUNKS, PITCH, Q8>(a, r.k, r.v, r.ks, r.vs, r.low, r.end, found, at, stage);
    }
    if (r.n % 32 == 0) {
        r.entry = r.next;
        r.next = entry_of(a, r, at + (32 + lane) * a.unit);
    }
    const int found = __shfl_sync(0xffffffffu, r.entry, r.n % 32);
    ++r.n;
    const int place = r.place;
    r.place += a.unit_in_page;
    if (r.place >= a.page_size) r.place -= a.page_size;
    // rows a fixed distance apart, which fits 32 bits
    const bool is_page = (uint32_t)found < (uint32_t)a.pages;
    const uint32_t entry = is_page ? (uint32_t)found : 0u, bits = is_page ? positions_of(r, at) : 0u;
    const uint32_t k_token = (uint32_t)a.k_token, v_token = (uint32_t)a.v_token;
    const char* k = r.k + (uint64_t)entry * (uint32_t)a.k_page + (uint64_t)(uint32_t)place * k_token;
    const char* v = r.v + (uint64_t)entry * (uint32_t)a.v_page + (uint64_t)(uint32_t)place * v_token;
    if constexpr (READING == kWhole) {
        const int row = lane / kLanes;
        k += (uint64_t)(uint32_t)row * k_token;
        v += (uint64_t)(uint32_t)row * v_token;
        const auto copy = [&](auto all) {                    // all: every row is there
#pragma unroll
            for (int i = 0; i < kTile / kRows; ++i) {
                const bool has = decltype(all)::value || ((bits >> (i * kRows + row)) & 1);
#pragma unroll
                for (int c0 = 0; c0 < CHUNKS; c0 += kLanes) {
                    const int c = c0 + (lane & (kLanes - 1));
                    if (CHUNKS % kLanes && c >= CHUNKS) continue;
                    const bool own = c * 16 < a.dim * ES;
                    const int piece = own ? c * 16 : 0;
                    const uint32_t dst = stage + (i * kRows + row) * PITCH + c * 16;
                    copy_async<16>(dst, k + (uint64_t)(uint32_t)(i * kRows) * k_token + piece, own && has);
                    copy_async<16>(dst + kTileBytes, v + (uint64_t)(uint32_t)(i * kRows) * v_token + piece, own && has);
                }
            }
        };
        if (bits == 0xffffu) copy(std::true_type());
        else copy(std::false_type());
    } else {
        ask_eights<CHUNKS, PITCH>(k, v, k_token, v_token, a.dim * ES / 8, bits, stage);
    }
    if constexpr (Q8) {
        const bool in = (bits >> (lane & 15)) & 1;
        const uint32_t token = entry * (uint32_t)a.page_size + (uint32_t)place + (in ? lane & 15 : 0);       // below 2^32 (a.whole_tiles)
        copy_async<4>(stage + 2 * kTileBytes + lane * 4, (lane < 16 ? r.ks : r.vs) + (uint64_t)token * (uint32_t)a.kv_heads, in);
    }
    return bits;
}

// The largest m of a head over the warps.
template <int HEADS> __device__ __forceinline__ float top_of(const float (*m)[HEADS], int head) {
    float top = m[0][head];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) top = fmaxf(top, m[w][head]);
    return top;
}

// ------------------------------------------------------------------------------------------------ matrix form
enum Kind { kBf16, kF16, kE4m3, kInt8 };

__device__ __forceinline__ void load_matrices(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void load_transposed(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ uint32_t transpose(uint32_t v) {
    uint32_t d;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(v));
    return d;
}
template <bool BF16> __device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if constexpr (BF16)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Two numbers as one register of 16-bit ones, the first in the low half.
template <bool BF16> __device__ __forceinline__ uint32_t pack2(float x, float y) {
    if constexpr (BF16) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(x, y);
        return *reinterpret_cast<const uint32_t*>(&v);
    } else {
        const __half2 v = __floats2half2_rn(x, y);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
}
template <bool BF16> __device__ __forceinline__ float2 unpack2(uint32_t v) {
    if constexpr (BF16) return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&v));
    else return __half22float2(*reinterpret_cast<const __half2*>(&v));
}
// Four 8-bit codes as two registers of two f16 numbers, exactly: bytes 0 and 1, bytes 2 and 3.
template <int KIND> __device__ __forceinline__ void widen(uint32_t four, uint32_t& low, uint32_t& high) {
    if constexpr (KIND == kE4m3) {
        asm("{.reg .b16 l, h; mov.b32 {l, h}, %2; cvt.rn.f16x2.e4m3x2 %0, l; cvt.rn.f16x2.e4m3x2 %1, h;}" : "=r"(low), "=r"(high) : "r"(four));
    } else {                                                 // 0x6400 + u is 1024 + u; u = code + 128
        const uint32_t u = four ^ 0x80808080u, x = __byte_perm(u, 0x64646464u, 0x4140), y = __byte_perm(u, 0x64646464u, 0x4342);
        const __half2 bias = __float2half2_rn(1152.0f);
        const __half2 p = __hsub2(*reinterpret_cast<const __half2*>(&x), bias), q = __hsub2(*reinterpret_cast<const __half2*>(&y), bias);
        low = *reinterpret_cast<const uint32_t*>(&p);
        high = *reinterpret_cast<const uint32_t*>(&q);
    }
}

// DT: width of a row in elements, rounded up; NT: tiles of eight heads.  LOW: p enters as two numbers; one is enough where p is f16 and
// the output bf16, whose own rounding is eight times as large.  QP: numbers to an element of q, two for
// floats (the second is what the rounding to f16 left).
template <int DT, int NT, int KIND, bool LOW, int QP> struct MmaCore {
    static constexpr bool kQ8 = KIND >= kE4m3, kIsBf16 = KIND == kBf16;
    static constexpr int kEs = kQ8 ? 1 : 2, kChunks = DT * kEs / 16, kPitch = 16 * (kChunks | 1), kTileBytes = kTile * kPitch;
    // Resident CTAs that the registers are cut for: by those that sums and q take.  8-bit rows of 128, four against three: 32 x 6000 64.6
    // and 66.1 us, in pages of one token 74.3 and 84.9, 33 x 12000 with 64 heads 122.3 and 120.7
    static constexpr int kHeld = DT * NT * (4 + 2 * QP) / 16, kCtas = kQ8 ? (kHeld <= 48 ? 4 : kHeld <= 64 ? 3 : 2) : kHeld <= 36 ? 3 : 1;
    static constexpr int kStage = 2 * kTileBytes + (kQ8 ? 128 : 0), kStages = DT <= 64 ? 3 : 2;
    static constexpr int kHeads = 8 * NT, kMergePitch = DT + 4;
    // 16-bit rows of 128: no more than two CTAs by their shared memory.  With three, or a third stage, the SMs' shares of the memory differ
    // so much that the last CTA ends 20 % behind the mean (64 x 8192: 254 us with two, 268 with three).
    static constexpr int kDim = DT, kLeastSmem = kQ8 || DT < 128 ? 0 : 77 * 1024;
    static constexpr bool kStagesQ = false;
    // p is at most 2^(kLift + kSlack): f16 numbers end at 65504, and below 2^-24 they are lost, which a p can be beside the largest one.
    // Over 8 bits p itself stays a float, and its product with the scale of a value is what f16 has to hold (`by`).
    static constexpr float kLift = KIND == kF16 ? 7.0f : 0.0f;
    static constexpr int kMostProduct = 15, kProduct = 6;    // powers of two: products stay below the one, the largest starts above the other
    static constexpr int kMostBy = 126;

    uint32_t q[DT / 16][NT][2][QP];
    // by head: the running maximum, kLift less it, the sum, what a product is multiplied with.  8 bits: m is a whole number, so that changes
    // of it are powers of two; `by`, a power of two, brings the products of p and their values' scales into f16
    float acc[DT / 16][NT][4], m[NT][2], c[NT][2], l[NT][2], f[NT][2], by[NT][2];
    bool far;                                                // a maximum of the warp's is so large that steps of floats show: every tile then changes them

    // q as the second operand of the scores: head g of each tile, two neighbouring dimensions to a register (16-bit caches), or four
    // to two registers (codes, as they lie in a lane's bytes).  Rows of q start where such an access may.
    __device__ __forceinline__ void begin(const AttnArgs& a, int r, int head0, int n_heads) {
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
        float factor[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            factor[nt] = a.scale;
            if constexpr (!kQ8) {
                const uint32_t* row = reinterpret_cast<const uint32_t*>(static_cast<const uint16_t*>(a.q) + r * a.q_row + (int64_t)(head0 + nt * 8 + g) * a.q_head) + t;
                const bool live = nt * 8 + g < n_heads;
#pragma unroll
                for (int j = 0; j < DT / 16; ++j)
#pragma unroll
                    for (int i = 0; i < 2; ++i) q[j][nt][i][0] = live && 16 * j + 8 * i + 2 * t < a.dim ? row[8 * j + 4 * i] : 0u;
            } else {
                const int64_t row = r * a.q_row + (int64_t)(head0 + nt * 8 + g) * a.q_head + 4 * t;
                const bool live = nt * 8 + g < n_heads;
                float4 x[DT / 16];
                if constexpr (QP == 2) {
#pragma unroll
                    for (int j = 0; j < DT / 16; ++j)
                        x[j] = live && 16 * j + 4 * t < a.dim ? *reinterpret_cast<const float4*>(static_cast<const float*>(a.q) + row + 16 * j) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                } else {
                    uint2 raw[DT / 16];
#pragma unroll
                    for (int j = 0; j < DT / 16; ++j)
                        raw[j] = live && 16 * j + 4 * t < a.dim ? *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(a.q) + row + 16 * j) : make_uint2(0u, 0u);
#pragma unroll
                    for (int j = 0; j < DT / 16; ++j) {
                        const float2 u = a.q_type == PP_F16 ? unpack2<false>(raw[j].x) : unpack2<true>(raw[j].x);
                        const float2 v = a.q_type == PP_F16 ? unpack2<false>(raw[j].y) : unpack2<true>(raw[j].y);
                        x[j] = make_float4(u.x, u.y, v.x, v.y);
                    }
                }
                float most = 0.0f, down = 1.0f;              // down: a power of two that brings the head's largest below 2, for f16 ends at 65504
                const auto finite = [](float v) { return fabsf(v) < INFINITY ? fabsf(v) : 0.0f; };
#pragma unroll
                for (int j = 0; j < DT / 16; ++j) most = fmaxf(fmaxf(fmaxf(most, finite(x[j].x)), fmaxf(finite(x[j].y), finite(x[j].z))), finite(x[j].w));
                most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
                most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
                if (most > 0.0f) {
                    const int e = min(max(((__float_as_int(most) >> 23) & 255) - 127, -126), 126);
                    down = __int_as_float((127 - e) << 23);
                    factor[nt] = a.scale * __int_as_float((127 + e) << 23);
                }
#pragma unroll
                for (int j = 0; j < DT / 16; ++j) {
                    const float4 v = make_float4(x[j].x * down, x[j].y * down, x[j].z * down, x[j].w * down);
                    q[j][nt][0][0] = pack2<false>(v.x, v.y);
                    q[j][nt][1][0] = pack2<false>(v.z, v.w);
                    if constexpr (QP == 2) {
                        const float2 u = unpack2<false>(q[j][nt][0][0]), w = unpack2<false>(q[j][nt][1][0]);
                        const auto rest = [](float a, float b) { return fabsf(b) == INFINITY ? 0.0f : a - b; };
                        q[j][nt][0][1] = pack2<false>(rest(v.x, u.x), rest(v.y, u.y));
                        q[j][nt][1][1] = pack2<false>(rest(v.z, w.x), rest(v.w, w.y));
                    }
                }
            }
#pragma unroll
            for (int j = 0; j < DT / 16; ++j)
#pragma unroll
                for (int k = 0; k < 4; ++k) acc[j][nt][k] = 0.0f;
        }
        far = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                f[nt][b] = __shfl_sync(0xffffffffu, factor[nt], (2 * t + b) * 4);
                m[nt][b] = kLowest;
                c[nt][b] = kLift - kLowest;
                l[nt][b] = 0.0f;
                by[nt][b] = power(kMostBy);
            }
    }

    __device__ __forceinline__ void tile(const AttnArgs& a, uint32_t stage, uint32_t bits) {
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
        float s[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[nt][i] = 0.0f;
        const uint32_t rows = stage + ((lane & 7) + ((lane >> 3) & 1) * 8) * kPitch + (lane >> 4) * 16;
        if constexpr (kQ8) {
#pragma unroll
            for (int c = 0; c < kChunks; c += 2) {
                uint32_t k[4];                               // rows g and g + 8 of one piece, then of the next
                load_matrices(k, rows + c * 16);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    uint32_t a0, a1, a2, a3;
                    widen<KIND>(k[2 * i], a0, a2);
                    widen<KIND>(k[2 * i + 1], a1, a3);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < QP; ++e) mma<kIsBf16>(s[nt], a0, a1, a2, a3, q[c + i][nt][0][e], q[c + i][nt][1][e]);
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < DT / 16; ++j) {
                uint32_t k[4];
                load_matrices(k, rows + j * 32);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mma<kIsBf16>(s[nt], k[0], k[1], k[2], k[3], q[j][nt][0][0], q[j][nt][1][0]);
            }
        }
        float v0 = 1.0f, v1 = 1.0f;                          // scales of the values at g and g + 8
        if constexpr (kQ8) {
            float k0, k1;
            const uint32_t at = stage + 2 * kTileBytes + g * 4;
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(k0) : "r"(at) : "memory");
            asm volatile("ld.shared.f32 %0, [%1+32];" : "=f"(k1) : "r"(at) : "memory");
            asm volatile("ld.shared.f32 %0, [%1+64];" : "=f"(v0) : "r"(at) : "memory");
            asm volatile("ld.shared.f32 %0, [%1+96];" : "=f"(v1) : "r"(at) : "memory");
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                s[nt][0] *= k0, s[nt][1] *= k0;
                s[nt][2] *= k1, s[nt][3] *= k1;
            }
        }
        const bool first = (bits >> g) & 1, second = (bits >> (g + 8)) & 1;
        float p[NT][4], x[NT][4];                            // p (logarithms first); the factors of the values' codes
        const auto exponents = [&](auto again) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    p[nt][i] = fmaf(s[nt][i], f[nt][i & 1], c[nt][i & 1]);
                    // A fused product has more bits than the maximum: their difference is up to half a step of the maximum, which from 2^20 on is
                    // no small part of a power of two, and from 2^27 on leaves f16 above or below.  Rounded products are on its steps.
                    if (decltype(again)::value && far) p[nt][i] = __fadd_rn(__fmul_rn(s[nt][i], f[nt][i & 1]), -m[nt][i & 1]) + kLift;
                }
            if (bits != 0xffffu) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!(i < 2 ? first : second)) p[nt][i] = -INFINITY;
            }
        };
        const auto products = [&] {                          // of p and the scales of its values
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    p[nt][i] = exp2_fast(p[nt][i]);
                    x[nt][i] = kQ8 ? p[nt][i] * (i < 2 ? v0 : v1) * by[nt][i & 1] : p[nt][i];
                }
        };
        exponents(std::false_type());
        float largest = p[0][0], heaviest = 0.0f;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) largest = fmaxf(largest, p[nt][i]);
        if constexpr (kQ8) {
            products();
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i) heaviest = fmaxf(heaviest, fabsf(x[nt][i]));
        }
        if (__any_sync(0xffffffffu, far || largest > kLift + kSlack || (kQ8 && heaviest >= power(kMostProduct)))) {
            int up[NT][2];                                   // by how many powers of two m rises (8 bits)
            bool large = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    float top = fmaxf(first ? s[nt][b] * f[nt][b] : kLowest, second ? s[nt][b + 2] * f[nt][b] : kLowest);
#pragma unroll
                    for (int o = 4; o < 32; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                    const float now = fmaxf(m[nt][b], kQ8 ? ceilf(top) : top);
                    if constexpr (kQ8) {
                        up[nt][b] = (int)fminf(now - m[nt][b], 512.0f);
                        l[nt][b] *= power(-up[nt][b]);
                    } else {
                        const float alpha = exp2_fast(m[nt][b] - now);
                        l[nt][b] *= alpha;
#pragma unroll
                        for (int j = 0; j < DT / 16; ++j) acc[j][nt][b] *= alpha, acc[j][nt][b + 2] *= alpha;
                    }
                    m[nt][b] = now;
                    c[nt][b] = kLift - now;
                    large |= fabsf(now) >= 0x1p20f && now != kLowest;
                }
            far = __any_sync(0xffffffffu, large);
            exponents(std::true_type());
            if constexpr (kQ8) {
                // by follows the largest product, not the largest scale: a large value at a position of no weight takes no bits from the others.
                // Products so far allow it to rise as m does; those of this tile may bring it down.
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        float top = fmaxf(fabsf(exp2_fast(p[nt][b]) * v0), fabsf(exp2_fast(p[nt][b + 2]) * v1));
#pragma unroll
                        for (int o = 4; o < 32; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                        const int held = exponent(by[nt][b]), may = min(held + up[nt][b], kMostBy), heavy = exponent(top);
                        const int now = heavy + may < kMostProduct ? may : max(kProduct - heavy, -126);
                        by[nt][b] = power(now);
                        const float change = power(now - held - up[nt][b]);       // 1 at most
#pragma unroll
                        for (int j = 0; j < DT / 16; ++j) acc[j][nt][b] *= change, acc[j][nt][b + 2] *= change;
                    }
                products();
            }
        }
        if constexpr (!kQ8) products();
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int b = 0; b < 2; ++b) l[nt][b] += p[nt][b] + p[nt][b + 2];
        uint32_t high[NT][2], low[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t h = pack2<kIsBf16>(x[nt][2 * i], x[nt][2 * i + 1]);
                const float2 back = unpack2<kIsBf16>(h);
                high[nt][i] = transpose(h);
                if constexpr (LOW) low[nt][i] = transpose(pack2<kIsBf16>(x[nt][2 * i] - back.x, x[nt][2 * i + 1] - back.y));
            }
        const uint32_t values = stage + kTileBytes;
        if constexpr (kQ8) {
            const uint32_t cols = values + ((lane & 7) + ((lane >> 3) & 1) * 8) * kPitch + (lane >> 4) * 16;
#pragma unroll
            for (int c = 0; c < kChunks; c += 2) {
                uint32_t v[4];                               // positions 0..7 and 8..15 of one piece, then of the next
                load_transposed(v, cols + c * 16);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    // bytes: dims 2g, 2g + 1 of position 2t, then of 2t + 1; row g of the product is dim 2g, row g + 8 dim 2g + 1
                    uint32_t a0, a1, a2, a3;
                    widen<KIND>(__byte_perm(v[2 * i], 0, 0x3120), a0, a1);
                    widen<KIND>(__byte_perm(v[2 * i + 1], 0, 0x3120), a2, a3);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        mma<kIsBf16>(acc[c + i][nt], a0, a1, a2, a3, high[nt][0], high[nt][1]);
                        if constexpr (LOW) mma<kIsBf16>(acc[c + i][nt], a0, a1, a2, a3, low[nt][0], low[nt][1]);
                    }
                }
            }
        } else {
            const uint32_t cols = values + ((lane & 7) + (lane >> 4) * 8) * kPitch + ((lane >> 3) & 1) * 16;
#pragma unroll
            for (int j = 0; j < DT / 16; ++j) {
                uint32_t v[4];
                load_transposed(v, cols + j * 32);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    mma<kIsBf16>(acc[j][nt], v[0], v[1], v[2], v[3], high[nt][0], high[nt][1]);
                    if constexpr (LOW) mma<kIsBf16>(acc[j][nt], v[0], v[1], v[2], v[3], low[nt][0], low[nt][1]);
                }
            }
        }
    }

    // m and l of this warp's positions, by head
    __device__ __forceinline__ void state(float* warp_m, float* warp_l) {
        const int lane = threadIdx.x & 31, t = lane & 3;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                float sum = l[nt][b];
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                if (lane < 4) {
                    warp_m[nt * 8 + 2 * t + b] = m[nt][b];
                    warp_l[nt * 8 + 2 * t + b] = sum;
                }
            }
    }
    // its sums, relative to the largest m of all warps or to its own
    __device__ __forceinline__ void sums(const float (*all)[kHeads], bool own, float* to) {
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const int head = nt * 8 + 2 * t + b;
                float weight = own ? 1.0f : weight_of(m[nt][b], top_of<kHeads>(all, head));
                if (kQ8) weight *= power(-exponent(by[nt][b]));
#pragma unroll
                for (int j = 0; j < DT / 16; ++j)
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        to[head * kMergePitch + 16 * j + (kQ8 ? 2 * g + i : g + 8 * i)] = acc[j][nt][b + 2 * i] * weight;
            }
    }
};

// ------------------------------------------------------------------------------------------------ scalar form
// DT: 64, 96, 128, 192, 256; HN: query heads of the chunk.  Rows of other types, and of any alignment, are read element by element and
// stored as floats, times their scale.
template <int DT, int HN> struct ScalarCore {
    // One tile on its way for each of many warps rather than several for few: 12 warps of 128 floats a row read 6.1 TB/s where 4 with three
    // tiles each read 5.2 (32 x 6000).
    static constexpr bool kQ8 = false;
    static constexpr int kEs = 4, kChunks = DT / 4, kPitch = 16 * (kChunks | 1), kTileBytes = kTile * kPitch;
    static constexpr int kHeads = HN, kMergePitch = DT;
    static constexpr int kStage = 2 * kTileBytes + 16 * 4 * HN, kStages = DT >= 128 ? 1 : 2;   // behind the rows: p by position and head
    static constexpr int kDim = DT, kCtas = 1, kLeastSmem = 0;
    static constexpr bool kStagesQ = true;
    static constexpr float kLift = 0.0f;

    float acc[DT / 32][HN], m[HN], l[HN];

    __device__ __forceinline__ void begin() {
#pragma unroll
        for (int h = 0; h < HN; ++h) {
            m[h] = kLowest;
            l[h] = 0.0f;
#pragma unroll
            for (int i = 0; i < DT / 32; ++i) acc[i][h] = 0.0f;
        }
    }

    // the next tile, element by element
    __device__ static uint32_t fetch(const AttnArgs& a, Reader& r, float* stage) {
        const int lane = threadIdx.x & 31, p = r.at + (lane & 15), entry = r.entry;
        const bool there = p >= r.low && p < r.end && (uint32_t)entry < (uint32_t)a.pages;
        const uint32_t bits = __ballot_sync(0xffffffffu, there) & 0xffffu;
        r.at += a.unit;
        r.entry = position_entry(a, r, r.at);
        int64_t off = 0;
        float scale = 1.0f;
        if (there) {
            const int place = p - (int)a.page.of((uint32_t)p) * a.page_size;
            off = lane < 16 ? (int64_t)entry * a.k_page + (int64_t)place * a.k_token : (int64_t)entry * a.v_page + (int64_t)place * a.v_token;
            if (a.ks) scale = (lane < 16 ? r.ks : r.vs)[((int64_t)entry * a.page_size + place) * a.kv_heads];
        }
        for (int row = 0; row < kTile; ++row) {
#pragma unroll
            for (int which = 0; which < 2; ++which) {
                const int64_t o = __shfl_sync(0xffffffffu, off, 16 * which + row);
                const float by = __shfl_sync(0xffffffffu, scale, 16 * which + row);
                const bool has = (bits >> row) & 1;
                const char* src = (which ? r.v : r.k) + o;
                float* dst = stage + (which * kTileBytes + row * kPitch) / 4;
#pragma unroll
                for (int i = 0; i < DT / 32; ++i) {
                    const int d = lane + 32 * i;
                    float x = 0.0f;
                    if (has && d < a.dim) {
                        if (a.type == PP_F32) x = reinterpret_cast<const float*>(src)[d];
                        else if (a.type == PP_F16) x = __half2float(reinterpret_cast<const __half*>(src)[d]);
                        else if (a.type == PP_BF16) x = __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(src)[d]);
                        else if (a.type == PP_E4M3) x = (float)reinterpret_cast<const __nv_fp8_e4m3*>(src)[d] * by;
                        else x = (float)reinterpret_cast<const int8_t*>(src)[d] * by;
                    }
                    dst[d] = x;
                }
            }
        }
        return bits;
    }

    __device__ __forceinline__ void tile(const AttnArgs& a, float* stage, uint32_t bits, const float* q) {
        const int lane = threadIdx.x & 31, key = lane & 15, half = lane >> 4;
        float s[HN];
#pragma unroll
        for (int h = 0; h < HN; ++h) s[h] = 0.0f;
        const float4* row = reinterpret_cast<const float4*>(stage + key * (kPitch / 4));
#pragma unroll 4
        for (int c = half; c < DT / 4; c += 2) {
            const float4 k = row[c];
#pragma unroll
            for (int h = 0; h < HN; ++h) {
                const float4 x = *reinterpret_cast<const float4*>(q + h * DT + 4 * c);
                s[h] = fmaf(k.x, x.x, fmaf(k.y, x.y, fmaf(k.z, x.z, fmaf(k.w, x.w, s[h]))));
            }
        }
        const bool there = (bits >> key) & 1;
        float* p = stage + 2 * kTileBytes / 4;
        bool higher = false;
#pragma unroll
        for (int h = 0; h < HN; ++h) {
            s[h] = (s[h] + __shfl_xor_sync(0xffffffffu, s[h], 16)) * a.scale;
            if (!there) s[h] = -INFINITY;
            higher |= s[h] - m[h] > kSlack;
        }
        if (__any_sync(0xffffffffu, higher)) {
#pragma unroll
            for (int h = 0; h < HN; ++h) {
                float top = s[h];
#pragma unroll
                for (int o = 1; o < 16; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                const float now = fmaxf(m[h], top), alpha = exp2_fast(m[h] - now);
                m[h] = now;
                l[h] *= alpha;
#pragma unroll
                for (int i = 0; i < DT / 32; ++i) acc[i][h] *= alpha;
            }
        }
#pragma unroll
        for (int h = 0; h < HN; ++h) {
            const float e = exp2_fast(s[h] - m[h]);
            l[h] += half ? 0.0f : e;
            if (!half) p[key * HN + h] = e;
        }
        __syncwarp();
        const float* v = stage + kTileBytes / 4 + lane;
#pragma unroll 4
        for (int j = 0; j < kTile; ++j) {
            float w[HN];
#pragma unroll
            for (int h = 0; h < HN; ++h) w[h] = p[j * HN + h];
#pragma unroll
            for (int i = 0; i < DT / 32; ++i) {
                const float x = v[j * (kPitch / 4) + 32 * i];
#pragma unroll
                for (int h = 0; h < HN; ++h) acc[i][h] = fmaf(w[h], x, acc[i][h]);
            }
        }
    }

    __device__ __forceinline__ void state(float* warp_m, float* warp_l) {
#pragma unroll
        for (int h = 0; h < HN; ++h) {
            float sum = l[h];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            if ((threadIdx.x & 31) == 0) {
                warp_m[h] = m[h];
                warp_l[h] = sum;
            }
        }
    }
    __device__ __forceinline__ void sums(const float (*all)[kHeads], bool own, float* to) {
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int h = 0; h < HN; ++h) {
            const float by = own ? 1.0f : weight_of(m[h], top_of<kHeads>(all, h));
#pragma unroll
            for (int i = 0; i < DT / 32; ++i) to[h * kMergePitch + lane + 32 * i] = acc[i][h] * by;
        }
    }
};

// ---------------------------------------------------------------------------------------------- one kernel for both
// Exclusive sums of the requests' units over the threads (a run of requests each), and the sum of all.
__device__ __forceinline__ int sum_before(int mine, int* warp_sums, int& all) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int up = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, up, o);
        if (lane >= o) up += x;
    }
    if (lane == 31) warp_sums[warp] = up;
    __syncthreads();
    int before = up - mine;
    all = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) before += warp_sums[w];
        all += warp_sums[w];
    }
    return before;
}

// u units cut into n parts, the first u % n of them one longer than the others: where part c starts, and the part of unit x.
struct Cut {
    int each, longer;
    __device__ __forceinline__ Cut(int u, int n) : each(u / n), longer(u - u / n * n) {}
    __device__ __forceinline__ int start(int c) const { return c * each + min(c, longer); }
    __device__ __forceinline__ int of(int x) const {
        const int edge = longer * (each + 1);
        return x < edge ? x / (each + 1) : longer + (x - edge) / each;
    }
};

// A head (chunk) whose units several CTAs share, noted by the first of them: in the place of the head among all (a.by_head), or where
// these are more than CTAs in that of the CTA, which can be the first one of one head only.
struct Note {
    int first, last;                                         // of the CTAs; last -1: no such head
    int row;                                                 // the first of out
    int rows;                                                // negative: the first one's part is the second of its two
};

// Thread-block clusters: a barrier in two halves, the second of which shows what others wrote before the first, and writes into another
// CTA's shared memory.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t at_rank(uint32_t own, int rank) {
    uint32_t d;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(d) : "r"(own), "r"(rank));
    return d;
}
__device__ __forceinline__ void store_remote(uint32_t at, float v) { asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(v) : "memory"); }
__device__ __forceinline__ void store_remote4(uint32_t at, float4 v) {
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1,%2,%3,%4};" ::"r"(at), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}

__device__ __forceinline__ float lse_of(float m, float l, float lift) { return l == 0.0f ? -INFINITY : (m - lift + log2f(l)) * kLn2; }

template <class Core, Reading READING> __global__ void __launch_bounds__(kThreads, Core::kCtas) attn_kernel(const __grid_constant__ AttnArgs a) {
    extern __shared__ __align__(128) unsigned char ring[];
    __shared__ int warp_sums[kWarps], found_base, found;
    __shared__ float warp_m[kWarps][Core::kHeads], warp_l[kWarps][Core::kHeads], all_m[Core::kHeads], all_l[Core::kHeads];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, c = blockIdx.x;
    pdl_release();
    if (a.cluster > 1) cluster_arrive();                     // awaited before the first write to another CTA's memory: it has started by then
    pdl_wait();

    const int per_request = (a.across ? a.kv_heads / kWarps : a.kv_heads) * a.n_chunks;
    int r, base = 0, u = 0, begin = 0, end = 1, ctas = 0, all = 0;    // unit u of the row of all, request r's from base on
    if (a.cluster) {
        r = c / a.cluster / per_request;
    } else {
        int mine = 0, before;
        int r0, r1;
        if (a.batch <= 32) {                                 // a request to a lane, in every warp: no barrier
            r0 = min(lane, a.batch), r1 = min(lane + 1, a.batch);
            if (lane < a.batch) mine = units_of(a, lane) * per_request;
            int up = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int x = __shfl_up_sync(0xffffffffu, up, o);
                if (lane >= o) up += x;
            }
            all = __shfl_sync(0xffffffffu, up, 31);
            before = up - mine;
        } else {
            const int each = (a.batch + kThreads - 1) / kThreads;
            r0 = min(tid * each, a.batch), r1 = min(r0 + each, a.batch);
            for (r = r0; r < r1; ++r) mine += units_of(a, r) * per_request;
            before = sum_before(mine, warp_sums, all);
        }
        ctas = min((int)gridDim.x, all);
        if (!a.by_head && tid == 0) reinterpret_cast<Note*>(a.ws)[c].last = -1;
        if (c >= ctas) return;
        const Cut cut(all, ctas);
        u = begin = cut.start(c);
        end = cut.start(c + 1);
        if (a.batch <= 32) {
            const int at = __ffs(__ballot_sync(0xffffffffu, u >= before && u < before + mine)) - 1;
            r = at;
            base = __shfl_sync(0xffffffffu, before, at);
        } else {
            if (u >= before && u < before + mine) {
                base = before;
                for (r = r0;; ++r) {
                    const int units = units_of(a, r) * per_request;
                    if (u < base + units) break;
                    base += units;
                }
                found = r;
                found_base = base;
            }
            __syncthreads();
            r = found;
            base = found_base;
        }
    }

    unsigned char* own = ring + warp * Core::kStages * Core::kStage;
    float* q = reinterpret_cast<float*>(ring + kWarps * Core::kStages * Core::kStage);
    float* merge = reinterpret_cast<float*>(ring);           // after the tiles, in their place: [warp][head][kMergePitch]
    while (u < end) {
        const int length = length_of(a, r), low = first_tile(a, length), units = units_of(a, r);
        int hc, t0, t1;
        if (a.cluster) {
            const int segment = c / a.cluster, rank = c - segment * a.cluster;
            const Cut cut(units, a.cluster);
            hc = segment - r * per_request;
            t0 = cut.start(rank);
            t1 = cut.start(rank + 1);
        } else {
            hc = (u - base) / units;
            t0 = u - base - hc * units;
            t1 = min(units, t0 + (end - u));
        }
        const int first_kv = hc / a.n_chunks * (a.across ? kWarps : 1), kv = a.across ? first_kv + warp : first_kv;
        const int head_in = hc % a.n_chunks * a.chunk, n_heads = min(a.chunk, a.group - head_in), head0 = kv * a.group + head_in;

        Reader reader;
        reader.k = a.k + kv * a.k_head;
        reader.v = a.v + kv * a.v_head;
        reader.ks = a.ks + kv;
        reader.vs = a.vs + kv;
        reader.row = a.table + r * a.ld_table;
        reader.low = first_position(a, length);
        reader.end = min(length, low + t1 * a.unit);
        reader.at = low + t0 * a.unit + (a.across ? 0 : warp * kTile);
        const int tiles = reader.at < reader.end ? (reader.end - reader.at + a.unit - 1) / a.unit : 0;
        start(a, reader);
        uint64_t there = 0;                                  // the rows that are there, 16 bits for each tile on its way, the last one's lowest
        int asked = 0, stage = 0;
        const auto request = [&]() {
            uint32_t bits = 0;
            if (asked < tiles) {
                if constexpr (READING != kElements) bits = ask<Core::kEs, Core::kChunks, Core::kPitch, Core::kQ8, READING>(a, reader, smem_at(own + stage * Core::kStage));
                else bits = Core::fetch(a, reader, reinterpret_cast<float*>(own + stage * Core::kStage));
            }
            there = there << 16 | bits;
            commit();
            ++asked;
            if (++stage == Core::kStages) stage = 0;
        };
        Core core;
        int at = 0;
#pragma unroll 1
        for (int i = 1 - Core::kStages;; ++i) {              // one call of request: its code is long
            if (i == 0) {
                if constexpr (Core::kStagesQ) {
                    stage_q<Core::kHeads, Core::kDim>(a, r, head0, n_heads, q);
                    __syncthreads();
                    core.begin();
                } else {
                    core.begin(a, r, head0, n_heads);
                }
            }
            if (i >= tiles) break;
            if (i >= 0) {
                if constexpr (Core::kStages > 1) wait_but<Core::kStages - 2>();
                __syncwarp();                                // this tile is here, and every lane has left the one before it
            }
            request();
            if (i < 0) continue;
            if constexpr (Core::kStages == 1) {
                wait_but<0>();
                __syncwarp();
            }
            const uint32_t bits = (uint32_t)(there >> (16 * (Core::kStages - 1))) & 0xffffu;
            if constexpr (Core::kStagesQ) core.tile(a, reinterpret_cast<float*>(own + at * Core::kStage), bits, q);
            else core.tile(a, smem_at(own + at * Core::kStage), bits);
            if (++at == Core::kStages) at = 0;
        }
        wait_but<0>();
        core.state(warp_m[warp], warp_l[warp]);
        __syncthreads();                                     // the ring is free, and every warp's m and l are known
        core.sums(warp_m, a.across, merge + warp * Core::kHeads * Core::kMergePitch);
        if (!a.across && tid < Core::kHeads) {
            const float top = top_of<Core::kHeads>(warp_m, tid);
            float sum = 0.0f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) sum += warp_l[w][tid] * weight_of(warp_m[w][tid], top);
            all_m[tid] = top;
            all_l[tid] = sum;
        }
        __syncthreads();
        const bool whole = t0 == 0 && t1 == units && a.cluster <= 1;
        const int64_t row0 = (int64_t)r * a.heads + first_kv * a.group + head_in;
        float* part = whole || a.cluster ? nullptr : a.ws + notes_floats(a.notes) + (2 * c + (u != begin)) * part_floats(a.part_rows, a.dim);
        constexpr int kFours = Core::kDim / 4;               // of a row
        // a cluster's CTAs share the rows' fours among them, round robin: each sends its part of a four to the CTA that joins it
        float4* inbox = reinterpret_cast<float4*>(ring + a.inbox);                             // [rank][its fours]
        float(*others)[2][Core::kHeads] = reinterpret_cast<float(*)[2][Core::kHeads]>(inbox + Core::kHeads * kFours + 8);   // [rank]: m and l
        const int rank = a.cluster > 1 ? c % a.cluster : 0, share = a.cluster > 1 ? (n_heads * kFours + a.cluster - 1) / a.cluster : 0;
        if (a.cluster > 1) cluster_wait();
        if (a.across) {                                      // a warp's rows are its own
#pragma unroll 1
            for (int i = lane; i < n_heads * kFours; i += 32) {
                const int h = i / kFours, d = 4 * (i - h * kFours);
                if (d >= a.dim) continue;
                const float4 sum = *reinterpret_cast<const float4*>(merge + (warp * Core::kHeads + h) * Core::kMergePitch + d);
                if (whole) store_out(a, row0 + warp * a.group + h, d, over(sum, warp_l[warp][h]));
                else *reinterpret_cast<float4*>(part + 2 * up4(a.part_rows) + (warp * a.chunk + h) * up4(a.dim) + d) = sum;
            }
        } else {
#pragma unroll 1
            for (int i = tid; i < n_heads * kFours; i += kThreads) {
                const int h = i / kFours, d = 4 * (i - h * kFours);
                if (d >= a.dim) continue;
                const float4* at = reinterpret_cast<const float4*>(merge + h * Core::kMergePitch + d);
                float4 sum = *at;
#pragma unroll
                for (int w = 1; w < kWarps; ++w) sum = add4(sum, at[w * Core::kHeads * Core::kMergePitch / 4]);
                if (whole) store_out(a, row0 + h, d, over(sum, all_l[h]));
                else if (part) *reinterpret_cast<float4*>(part + 2 * up4(a.part_rows) + h * up4(a.dim) + d) = sum;
                else store_remote4(at_rank(smem_at(inbox + rank * share + i / a.cluster), i % a.cluster), sum);
            }
        }
        if (part) {
            if (t0 == 0 && tid == 0)
                reinterpret_cast<Note*>(a.ws)[a.by_head ? r * per_request + hc : c] = {c, Cut(all, ctas).of(base + (hc + 1) * units - 1), (int)row0, u != begin ? -n_heads : n_heads};
        } else if (whole && a.by_head && !a.cluster && tid == 0) {
            reinterpret_cast<Note*>(a.ws)[r * per_request + hc].last = -1;
        }
        if (part || (whole && a.lse)) {
            const int w = a.across ? tid / n_heads : 0, h = tid - w * n_heads;
            if (w < (a.across ? kWarps : 1) && h < n_heads) {
                const float m = a.across ? warp_m[w][h] : all_m[h], l = a.across ? warp_l[w][h] : all_l[h];
                if (part) {
                    part[w * a.chunk + h] = m;
                    part[up4(a.part_rows) + w * a.chunk + h] = l;
                } else {
                    a.lse[row0 + w * a.group + h] = lse_of(m, l, Core::kLift);
                }
            }
        }
        if (a.cluster) {
            if (a.cluster == 1) return;
#pragma unroll 1
            for (int i = tid; i < a.cluster * n_heads; i += kThreads) {
                const int to = i / n_heads, h = i - to * n_heads;
                store_remote(at_rank(smem_at(&others[rank][0][h]), to), all_m[h]);
                store_remote(at_rank(smem_at(&others[rank][1][h]), to), all_l[h]);
            }
            cluster_arrive();
            cluster_wait();
#pragma unroll 1
            for (int n = tid; n < share; n += kThreads) {
                const int i = n * a.cluster + rank, h = i / kFours, d = 4 * (i - h * kFours);
                if (h >= n_heads || d >= a.dim) continue;
                float top = kLowest, l = 0.0f;
#pragma unroll 1
                for (int k = 0; k < a.cluster; ++k) top = fmaxf(top, others[k][0][h]);
                float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 2
                for (int k = 0; k < a.cluster; ++k) {
                    const float w = weight_of(others[k][0][h], top);
                    l = fmaf(others[k][1][h], w, l);
                    sum = fma4(inbox[k * share + n], w, sum);
                }
                store_out(a, row0 + h, d, over(sum, l));
                if (a.lse && d == 0) a.lse[row0 + h] = lse_of(top, l, Core::kLift);
            }
            return;
        }
        __syncthreads();
        u += t1 - t0;
        if (u == base + units * per_request) {
            base = u;
            ++r;
        }
    }
}

// ------------------------------------------------------------------------------------------------------ forms
using Kernel = void (*)(const AttnArgs);
struct Form {
    Kernel kernel = nullptr;
    int smem = 0, inbox = 0, heads = 0;
    float lift = 0.0f;
    bool shares_q = false;
    PerDeviceOnce* opt_in = nullptr;
    int (*resident)[4] = nullptr;                            // clusters of 1, 2, 4 and 8 CTAs that a device holds, by device
};

template <class Core, Reading READING> Form form_of() {
    static PerDeviceOnce opt_in;
    static int resident[PerDeviceOnce::kMaxDevices][4] = {};
    Form f;
    f.kernel = attn_kernel<Core, READING>;
    f.inbox = std::max(kWarps * Core::kStages * Core::kStage, kWarps * Core::kHeads * Core::kMergePitch * 4) + (Core::kStagesQ ? Core::kHeads * Core::kDim * 4 : 0);
    f.smem = std::max(Core::kLeastSmem, f.inbox + Core::kHeads * Core::kDim * 4 + 8 * 16 + 8 * 2 * Core::kHeads * 4);    // shares are rounded up for each rank
    f.heads = Core::kHeads;
    f.lift = Core::kLift;
    f.shares_q = Core::kStagesQ;
    f.opt_in = &opt_in;
    f.resident = resident;
    return f;
}
// The forms by the cache's type, each compiled in a file of its own.  dim: of a row; two: 16 query heads instead of 8; reading: of rows.
Form form_bf16(Reading reading, int dim, bool two);
Form form_f16(Reading reading, int dim, bool two);
Form form_e4m3(Reading reading, pp_dtype_t q_type, int dim, bool two);
Form form_int8(Reading reading, pp_dtype_t q_type, int dim, bool two);
Form form_scalar(Reading reading, int dim, int group);

template <int KIND, bool LOW, int QP, Reading READING> Form mma_form(int dim, bool two) {
    if constexpr (QP == 1)
        if (two) return dim <= 64 ? form_of<MmaCore<64, 2, KIND, LOW, QP>, READING>() : dim <= 96 ? form_of<MmaCore<96, 2, KIND, LOW, QP>, READING>() : form_of<MmaCore<128, 2, KIND, LOW, QP>, READING>();
    return dim <= 64 ? form_of<MmaCore<64, 1, KIND, LOW, QP>, READING>() : dim <= 96 ? form_of<MmaCore<96, 1, KIND, LOW, QP>, READING>()
         : dim <= 128 ? form_of<MmaCore<128, 1, KIND, LOW, QP>, READING>() : dim <= 192 ? form_of<MmaCore<192, 1, KIND, LOW, QP>, READING>() : form_of<MmaCore<256, 1, KIND, LOW, QP>, READING>();
}
template <int KIND, bool LOW, int QP> Form mma_form(Reading reading, int dim, bool two) {
    return reading == kWhole ? mma_form<KIND, LOW, QP, kWhole>(dim, two) : mma_form<KIND, LOW, QP, kRows>(dim, two);
}
template <int KIND> Form mma_form8(Reading reading, pp_dtype_t q_type, int dim, bool two) {
    return q_type == PP_BF16 ? mma_form<KIND, false, 1>(reading, dim, two) : q_type == PP_F16 ? mma_form<KIND, true, 1>(reading, dim, two) : mma_form<KIND, true, 2>(reading, dim, false);
}
template <Reading READING> Form scalar_form(int dim, int group) {
    const auto of = [&](auto d) {
        constexpr int DT = decltype(d)::value;
        return group <= 1 ? form_of<ScalarCore<DT, 1>, READING>() : group <= 4 ? form_of<ScalarCore<DT, 4>, READING>() : form_of<ScalarCore<DT, 8>, READING>();
    };
    if (dim <= 64) return of(std::integral_constant<int, 64>());
    if (dim <= 96) return of(std::integral_constant<int, 96>());
    if (dim <= 128) return of(std::integral_constant<int, 128>());
    return dim <= 192 ? of(std::integral_constant<int, 192>()) : of(std::integral_constant<int, 256>());
}

}  // namespace attn
}  // namespace pp
