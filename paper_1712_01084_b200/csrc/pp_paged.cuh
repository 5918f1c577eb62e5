// What the operators of the paged key-value cache share (pp_paged.cu, pp_attn.cu): division by a number that the host knows,
// the checks of a cache's description, rows that must not overlap.
#pragma once
#include <algorithm>

#include "pp_decode.cuh"

namespace pp {

// n / d for 0 <= n < 2^31 by one multiplication: m = ceil(2^p / d) with p = 31 + ceil(log2 d) exceeds 2^p / d by e / d, e < d <= 2^(p-31),
// so n m / 2^p exceeds n / d by n e / (d 2^p) < 1 / d, which never reaches the next whole number.
struct Divisor {
    uint32_t d = 1, m = 0, p = 31;
    Divisor() = default;
    explicit Divisor(uint32_t by) : d(by) {
        uint32_t log = 0;
        while ((1ull << log) < by) ++log;
        p = 31 + log;
        m = (uint32_t)(((1ull << p) + by - 1) / by);         // < 2^32: 2^p / d < 2^32 for d > 2^(log-1), and 2^31 for d = 1
    }
#ifdef __CUDACC__
    __device__ __forceinline__ uint32_t of(uint32_t n) const { return (uint32_t)(((uint64_t)n * m) >> p); }
#endif
};

constexpr int kMaxHeadDim = 256;

// Two rows of a strided array [n0][n1][n2][width] share no element: from the smallest stride up, each is at least what the axes
// below it span.  (Axes of one entry do not count.)
inline bool rows_apart(int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t n2, int64_t s2, int64_t width) {
    std::pair<int64_t, int64_t> axis[3] = {{s0, n0}, {s1, n1}, {s2, n2}};
    std::sort(axis, axis + 3);
    int64_t span = width;
    for (const auto& [stride, n] : axis) {
        if (n <= 1) continue;
        if (stride < span) return false;
        span += stride * (n - 1);
    }
    return true;
}

// Whether the spans of two arrays meet (bytes; nothing meets an absent or empty one).
inline bool spans_meet(const void* p, int64_t n, const void* q, int64_t m) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
    return p && q && n > 0 && m > 0 && a < b + (uint64_t)m && b < a + (uint64_t)n;
}
// Rows of a strided array [n0][n1][n2][width] that are apart (rows_apart), in bytes: its axes of several entries, the largest stride first.
struct Rows {
    uintptr_t at;
    int64_t width, stride[3], count[3];
    int axes = 0;
    Rows(const void* p, int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t n2, int64_t s2, int64_t elements, int bytes)
        : at(reinterpret_cast<uintptr_t>(p)), width(elements * bytes) {
        std::pair<int64_t, int64_t> axis[3] = {{s0, n0}, {s1, n1}, {s2, n2}};
        if (axis[0] < axis[1]) std::swap(axis[0], axis[1]);
        if (axis[1] < axis[2]) std::swap(axis[1], axis[2]);
        if (axis[0] < axis[1]) std::swap(axis[0], axis[1]);
        for (const auto& [s, n] : axis)
            if (n > 1) stride[axes] = s * bytes, count[axes++] = n;
    }
    int64_t span(int axis = 0) const {                       // of the axes from this one on
        int64_t n = width;
        for (int i = axis; i < axes; ++i) n += stride[i] * (count[i] - 1);
        return n;
    }
    // Whether bytes from .. to - 1, counted from the start of axis `axis`, hold some of a row's.
    bool meet(int64_t from, int64_t to, int axis = 0) const {
        if (from >= to || to <= 0 || from >= span(axis)) return false;
        if (axis == axes) return true;
        const int64_t s = stride[axis], inner = span(axis + 1);
        const int64_t first = from < inner ? 0 : (from - inner) / s + 1, last = std::min(count[axis] - 1, (to - 1) / s);
        if (last - first > 1) return true;                   // one between them lies inside as a whole
        for (int64_t i = first; i <= last; ++i)
            if (meet(from - i * s, to - i * s, axis + 1)) return true;
        return false;
    }
    bool meet(const void* p, int64_t n) const {
        if (!p || n <= 0 || !spans_meet(p, n, reinterpret_cast<const void*>(at), span())) return false;
        const int64_t from = (int64_t)(reinterpret_cast<uintptr_t>(p) - at);
        return meet(from, from + n);
    }
    // Whether rows of another array with the same axes, d bytes behind, share bytes with these: d is, but for less than a row, a sum of
    // differences of places, of which each axis leaves two to choose from.
    bool meet_shifted(int64_t d, int axis = 0) const {
        if (axis == axes) return d < width && -d < width;
        const int64_t s = stride[axis], near = d >= 0 ? d / s : -((-d + s - 1) / s);
        for (int64_t i = near; i <= near + 1; ++i)
            if (i < count[axis] && -i < count[axis] && meet_shifted(d - i * s, axis + 1)) return true;
        return false;
    }
    bool meet(const Rows& other) const {                     // arrays of other strides in each other's range count as apart
        if (axes != other.axes || width != other.width) return false;
        for (int i = 0; i < axes; ++i)
            if (stride[i] != other.stride[i] || count[i] != other.count[i]) return false;
        return meet_shifted((int64_t)(other.at - at));
    }
};
inline Rows rows_of_keys(const pp_paged_cache_t& c) {
    return Rows(c.k, c.pages, c.k_page, c.page_size, c.k_token, c.kv_heads, c.k_head, c.head_dim, type_bytes(c.dtype));
}
inline Rows rows_of_values(const pp_paged_cache_t& c) {
    return Rows(c.v, c.pages, c.v_page, c.page_size, c.v_token, c.kv_heads, c.v_head, c.head_dim, type_bytes(c.dtype));
}
inline int64_t scales_bytes(const pp_paged_cache_t& c) { return 4 * (int64_t)c.pages * c.page_size * c.kv_heads; }

// What a cache holds: rows of keys and values, scales; what lies between rows is not the cache's.  Whether an array shares bytes with it.
struct Held {
    Rows k, v;
    const float *k_scales, *v_scales;
    int64_t scales;
    explicit Held(const pp_paged_cache_t& c) : k(rows_of_keys(c)), v(rows_of_values(c)), k_scales(c.k_scales), v_scales(c.v_scales), scales(scales_bytes(c)) {}
    bool meet(const void* p, int64_t n) const {
        return k.meet(p, n) || v.meet(p, n) || spans_meet(p, n, k_scales, scales) || spans_meet(p, n, v_scales, scales);
    }
};

// What is wrong with a cache's description, if anything.
inline pp_status_t check_cache(const pp_paged_cache_t* c) {
    if (!c || !c->k || !c->v || c->k == c->v || c->pages < 1 || c->page_size < 1 || c->kv_heads < 1 || c->head_dim < 1) return PP_ERR_INVALID_ARG;
    if (!is_float(c->dtype) && !is_8bit(c->dtype)) return PP_ERR_UNSUPPORTED;
    if (c->head_dim > kMaxHeadDim || c->page_size > (1 << 20) || (int64_t)c->pages * c->page_size > (int64_t)1 << 40 || c->kv_heads > (1 << 16))
        return PP_ERR_UNSUPPORTED;
    if (is_8bit(c->dtype) != (c->k_scales != nullptr) || is_8bit(c->dtype) != (c->v_scales != nullptr) || (c->k_scales && c->k_scales == c->v_scales))
        return PP_ERR_INVALID_ARG;
    const size_t tb = (size_t)type_bytes(c->dtype);
    if (!aligned_to(c->k, tb) || !aligned_to(c->v, tb) || !aligned_to(c->k_scales, 4) || !aligned_to(c->v_scales, 4)) return PP_ERR_INVALID_ARG;
    const int64_t most = (int64_t)1 << 56;                   // no sum of offsets passes 63 bits
    for (const int64_t s : {c->k_page, c->k_token, c->k_head, c->v_page, c->v_token, c->v_head})
        if (s < 0 || s > most) return PP_ERR_INVALID_ARG;
    for (const int64_t s : {c->k_page, c->v_page})
        if (s > most / c->pages) return PP_ERR_INVALID_ARG;
    for (const int64_t s : {c->k_token, c->v_token})
        if (s > most / c->page_size) return PP_ERR_INVALID_ARG;
    for (const int64_t s : {c->k_head, c->v_head})
        if (s > most / c->kv_heads) return PP_ERR_INVALID_ARG;
    if (!rows_apart(c->pages, c->k_page, c->page_size, c->k_token, c->kv_heads, c->k_head, c->head_dim) ||
        !rows_apart(c->pages, c->v_page, c->page_size, c->v_token, c->kv_heads, c->v_head, c->head_dim)) return PP_ERR_INVALID_ARG;
    const Held held(*c);
    if (held.k.meet(held.v) || spans_meet(c->k_scales, held.scales, c->v_scales, held.scales)) return PP_ERR_INVALID_ARG;
    for (const float* s : {c->k_scales, c->v_scales})
        if (held.k.meet(s, held.scales) || held.v.meet(s, held.scales)) return PP_ERR_INVALID_ARG;
    return PP_OK;
}

// The largest of 16, 8, 4, 2, 1 that divides every start of a row, in bytes: axes of one entry do not count.
inline int row_alignment(const void* p, int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t n2, int64_t s2, int bytes) {
    uint64_t bits = reinterpret_cast<uintptr_t>(p);
    if (n0 > 1) bits |= (uint64_t)(s0 * bytes);
    if (n1 > 1) bits |= (uint64_t)(s1 * bytes);
    if (n2 > 1) bits |= (uint64_t)(s2 * bytes);
    int a = 16;
    while (bits & (uint64_t)(a - 1)) a /= 2;
    return a;
}
inline int cache_alignment(const pp_paged_cache_t& c) {
    const int tb = type_bytes(c.dtype);
    return std::min(row_alignment(c.k, c.pages, c.k_page, c.page_size, c.k_token, c.kv_heads, c.k_head, tb),
                    row_alignment(c.v, c.pages, c.v_page, c.page_size, c.v_token, c.kv_heads, c.v_head, tb));
}

}  // namespace pp
