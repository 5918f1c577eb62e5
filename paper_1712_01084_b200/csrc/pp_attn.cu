// Attention over a paged key-value cache: the kernel that joins parts, the choice of form and division, and the C interface.
#include "pp_attn.cuh"

#include <mutex>

namespace pp {
namespace attn {
namespace {

// Joins the parts of the head (chunk) of note blockIdx.x, if there is one.  CTA blockIdx.y takes a share of its rows and, of their
// dimensions, one of SLICES.  As many warps to a row as there are, and as many parts at once to a warp as there are slices: few
// heads of many parts are joined by many CTAs.  One pass, with a running maximum for each warp and part at once.
constexpr int kJoinWarps = 8, kJoinThreads = kJoinWarps * 32;
template <int SLICES> __global__ void __launch_bounds__(kJoinThreads) join_kernel(const __grid_constant__ AttnArgs a, float lift) {
    __shared__ float4 sums[kJoinWarps][kMaxHeadDim / 4];
    __shared__ float ls[kJoinWarps], tops[kJoinWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, step = gridDim.y / SLICES, share = blockIdx.y / SLICES, slice = blockIdx.y % SLICES;
    pdl_release();
    pdl_wait();
    const int4 raw = __ldcg(reinterpret_cast<const int4*>(a.ws) + blockIdx.x);
    const Note note{raw.x, raw.y, raw.z, raw.w};
    if (note.last < 0) return;
    const int64_t floats = part_floats(a.part_rows, a.dim), second = note.rows < 0 ? floats : 0;
    const float* parts = a.ws + notes_floats(a.notes);
    const auto part = [&](int c) { return parts + 2 * c * floats + (c == note.first ? second : 0); };     // read past L1: written by other SMs
    const int rows4 = up4(a.part_rows), dim4 = up4(a.dim), n_heads = abs(note.rows), all_rows = n_heads * (a.across ? kWarps : 1);
    const int rows = (all_rows - share + step - 1) / step;   // of this CTA
    if (rows < 1) return;
    // a part takes 32 / SLICES lanes, up to two fours of dimensions each
    constexpr int lanes = 32 / SLICES;
    const int column = lane % lanes, group = lane / lanes, fours = (dim4 / 4 + SLICES - 1) / SLICES, first4 = slice * fours;
    const int at_once = min(rows, kJoinWarps), per = kJoinWarps / at_once, sub = warp % per;
    for (int done = 0; done < rows; done += at_once) {
        const int n = done + warp / per, row = share + n * step, head = row / n_heads;        // head: of the four (across)
        const bool live = warp / per < at_once && n < rows;
        const int h = head * a.chunk + row - head * n_heads;
        const int64_t to = (int64_t)note.row + head * a.group + row - head * n_heads;
        float top = kLowest, l = 0.0f;
        float4 acc[2] = {make_float4(0.0f, 0.0f, 0.0f, 0.0f), make_float4(0.0f, 0.0f, 0.0f, 0.0f)};
        if (live) {
#pragma unroll 4
            for (int c = note.first + sub * SLICES + group; c <= note.last; c += per * SLICES) {
                const float* p = part(c);
                const float4* x = reinterpret_cast<const float4*>(p + 2 * rows4 + h * dim4) + first4 + column;
                const float m = __ldcg(p + h), sum = __ldcg(p + rows4 + h), now = fmaxf(top, m), before = weight_of(top, now), w = weight_of(m, now);
                l = fmaf(l, before, sum * w);
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    if (column + lanes * i < fours && 4 * (first4 + column + lanes * i) < a.dim) {
                        const float4 v = __ldcg(x + lanes * i);
                        acc[i] = fma4(v, w, make_float4(acc[i].x * before, acc[i].y * before, acc[i].z * before, acc[i].w * before));
                    }
                top = now;
            }
#pragma unroll
            for (int o = lanes; o < 32; o <<= 1) {
                const float m = __shfl_xor_sync(0xffffffffu, top, o), now = fmaxf(top, m), mine = weight_of(top, now), w = weight_of(m, now);
                l = fmaf(l, mine, __shfl_xor_sync(0xffffffffu, l, o) * w);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float4 v = make_float4(__shfl_xor_sync(0xffffffffu, acc[i].x, o), __shfl_xor_sync(0xffffffffu, acc[i].y, o),
                                                 __shfl_xor_sync(0xffffffffu, acc[i].z, o), __shfl_xor_sync(0xffffffffu, acc[i].w, o));
                    acc[i] = fma4(v, w, make_float4(acc[i].x * mine, acc[i].y * mine, acc[i].z * mine, acc[i].w * mine));
                }
                top = now;
            }
        }
        if (group == 0) {
#pragma unroll
            for (int i = 0; i < 2; ++i) sums[warp][column + lanes * i] = acc[i];
        }
        if (lane == 0) {
            ls[warp] = l;
            tops[warp] = top;
        }
        __syncthreads();
        if (live && sub == 0) {
            for (int w = 1; w < per; ++w) top = fmaxf(top, tops[warp + w]);
            l = 0.0f;
            for (int w = 0; w < per; ++w) l = fmaf(ls[warp + w], weight_of(tops[warp + w], top), l);
            for (int f = lane; f < fours && 4 * (first4 + f) < a.dim; f += 32) {
                float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                for (int w = 0; w < per; ++w) sum = fma4(sums[warp + w][f], weight_of(tops[warp + w], top), sum);
                store_out(a, to, 4 * (first4 + f), over(sum, l));
            }
            if (a.lse && lane == 0 && slice == 0) a.lse[to] = lse_of(top, l, lift);
        }
        __syncthreads();
    }
}

// The form of a call.
struct Choice {
    Form form;
    Reading reading;
    int granule, chunk;                                      // bytes of an asynchronous copy; query heads of a CTA
    bool whole;                                              // whole tiles (AttnArgs)
};
// q_on: what divides the starts of q's rows, in bytes.
Choice choose(const pp_paged_cache_t& c, pp_dtype_t q_type, int q_on, int group) {
    const int es = type_bytes(c.dtype), row = c.head_dim * es;
    int granule = std::min(cache_alignment(c), 16);
    while (row % granule) granule /= 2;
    const int64_t far = std::max({c.k_page, c.k_token, c.v_page, c.v_token}) * es;
    const bool whole = c.page_size % kTile == 0 && granule >= 8 && far <= UINT32_MAX && (int64_t)c.pages * c.page_size <= UINT32_MAX;
    const Reading reading = granule < 4 ? kElements : whole && granule == 16 ? kWhole : kRows;
    if (reading != kElements && c.dtype != PP_F32 && q_on >= (!is_8bit(c.dtype) ? 4 : q_type == PP_F32 ? 16 : 8)) {
        // 16 heads where a key-value head has more than 8: above 128 dimensions, or with q as two numbers, they do not fit the registers
        const bool two = group > 8 && c.head_dim <= 128 && (!is_8bit(c.dtype) || q_type != PP_F32);
        const Form f = c.dtype == PP_BF16 ? form_bf16(reading, c.head_dim, two) : c.dtype == PP_F16 ? form_f16(reading, c.head_dim, two)
                     : c.dtype == PP_E4M3 ? form_e4m3(reading, q_type, c.head_dim, two) : form_int8(reading, q_type, c.head_dim, two);
        return {f, reading, granule, two ? 16 : 8, whole};
    }
    const Reading own = c.dtype == PP_F32 ? reading : kElements;
    const Form f = form_scalar(own, c.head_dim, group);
    return {f, own, granule, f.heads, whole && own != kElements};
}

// Clusters of 1, 2, 4 and 8 CTAs that the current device holds at once.  A cluster keeps to one group of SMs, so those of eight are fewer
// than an eighth of the CTAs: 36 of them, for which there were CTAs enough, took two rounds (9 x 1000, heads of 256: 17 us).
cudaError_t hold(const Form& f, int (&n)[4]) {
    int device = 0;
    if (cudaError_t e = cudaGetDevice(&device)) return e;
    static std::mutex first;                                 // of two first calls at once the second reads what the first one found
    const std::lock_guard<std::mutex> one(first);
    if (f.opt_in->is_done(device)) {
        for (int i = 0; i < 4; ++i) n[i] = f.resident[device][i];
        return cudaSuccess;
    }
    if (cudaError_t e = cudaFuncSetAttribute(f.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, f.smem)) return e;
    // An SM divides its memory between L1 and shared memory as its kernels ask, and changes that only when it is empty: with the second
    // kernel's smaller wish in force the last of the CTAs would start when others end.
    for (const void* k : {reinterpret_cast<const void*>(f.kernel), reinterpret_cast<const void*>(join_kernel<1>), reinterpret_cast<const void*>(join_kernel<2>),
                          reinterpret_cast<const void*>(join_kernel<4>)})
        if (cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared)) return e;
    int each = 0;
    if (cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&each, f.kernel, kThreads, (size_t)f.smem)) return e;
    n[0] = std::max(each, 1) * sm_count();
    for (int i = 1; i < 4; ++i) {
        cudaLaunchAttribute at{};
        at.id = cudaLaunchAttributeClusterDimension;
        at.val.clusterDim.x = 1u << i;
        at.val.clusterDim.y = at.val.clusterDim.z = 1;
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3(1u << i);
        cfg.blockDim = dim3(kThreads);
        cfg.dynamicSmemBytes = (size_t)f.smem;
        cfg.attrs = &at;
        cfg.numAttrs = 1;
        if (cudaError_t e = cudaOccupancyMaxActiveClusters(&n[i], f.kernel, &cfg)) return e;
    }
    if (device < PerDeviceOnce::kMaxDevices) {
        for (int i = 0; i < 4; ++i) f.resident[device][i] = n[i];
        f.opt_in->mark(device);
    }
    return cudaSuccess;
}

pp_status_t check_call(const pp_paged_cache_t* cache, pp_dtype_t q_type, int batch, int heads, int width, int window) {
    if (const pp_status_t st = check_cache(cache)) return st;
    if (!is_float(q_type) || (q_type != cache->dtype && !is_8bit(cache->dtype))) return PP_ERR_UNSUPPORTED;
    if (batch < 0 || heads < 1 || heads % cache->kv_heads || width < 1 || window < 0) return PP_ERR_INVALID_ARG;
    const int64_t capacity = (int64_t)width * cache->page_size;
    // positions are 32 bits, and entries are looked up 63 units ahead of a tile (Reader)
    if (capacity > INT32_MAX - kAheadMost || heads > (1 << 20) || (int64_t)batch * heads > INT32_MAX) return PP_ERR_UNSUPPORTED;
    if ((int64_t)batch * heads > INT32_MAX / (capacity / kUnit + 2)) return PP_ERR_UNSUPPORTED;     // units are counted in 32 bits
    return PP_OK;
}

// How a call is divided.
struct Division {
    int grid, cluster;                                       // cluster 0: equal parts of all units, joined by a second kernel
    bool across;                                             // of four heads at once
    int notes, part_rows;
    int64_t bytes;                                           // of workspace
};
// Costs in units of 64 positions to a CTA, some 0.6 us while latency rules (twice that in the scalar form), going by the table's
// width.  Equal parts of all units: sums over lengths, the workspace and a second kernel, 4 us, and CTAs that share their SM with as
// many others as it holds.  A CTA or a cluster of up to eight to each head (chunk): as many rounds as the GPU needs for them, each a
// CTA's share and 2 us for its start and end; a cluster's exchange costs 2.3 us; and a 32nd of a long share, since heads that do not
// fill the GPU leave memory idle.  With 10 for equal parts and no 32nd: 2 x 3000, heads of 64, 11.5 us for 8.7 now, 23 x 1025 in 8
// bits 17.6 for 15.3, 12 x 1500 with 16-bit heads of 256 30.1 for 32.2; with 12 and no 32nd 30 x 3000 bf16 57.7 for 52.0.
constexpr int kEqualParts = 12, kRound = 3, kExchange = 4;
Division divide(const pp_paged_cache_t& c, const Form& f, int batch, int width, int window, int chunk, int n_chunks, const int (&held)[4]) {
    const int resident = held[0];
    const bool fours = c.kv_heads % kWarps == 0 && !f.shares_q;
    const int64_t capacity = (int64_t)width * c.page_size, longest = window > 0 ? std::min<int64_t>((int64_t)window + kTile - 1, capacity) : capacity;
    const int64_t units = std::max<int64_t>(1, (longest + kUnit - 1) / kUnit), heads = (int64_t)batch * c.kv_heads * n_chunks;
    const int64_t weight = f.shares_q ? 2 : 1;
    int64_t least = weight * (heads * units / resident + 1) + kEqualParts, best = 0;
    for (int i = 0; i < 4; ++i) {
        const int64_t cluster = 1 << i, rounds = held[i] ? (heads + held[i] - 1) / held[i] : INT32_MAX, own = (units + cluster - 1) / cluster;
        const int64_t cost = rounds * (weight * own + own / 32 + kRound + (cluster > 1 ? kExchange : 0));
        if (cost < least && heads * cluster <= INT32_MAX) least = cost, best = cluster;
    }
    if (units == 1 && best != 1) {                           // nothing to divide
        best = 1;
        least = (heads + resident - 1) / resident * (weight + kRound);
    }
    if (fours && best != 0) {                                // short heads, more than the GPU holds: a warp to each, four to a CTA
        const int64_t cost = (heads / kWarps + resident - 1) / resident * (kWarps * units + kRound);
        if (cost < least) return {(int)(heads / kWarps), 1, true, 0, 0, 0};
    }
    if (best) return {(int)(heads * best), (int)best, false, 0, 0, 0};
    // Four neighbouring heads at once where the scales of their rows share lines of memory, or their rows do: where heads lie side by side
    // and a row is no multiple of 256 bytes, heads read one after another fetch the lines between them twice (32 x 6000, eight
    // heads of 72 / 96: 88 / 98 us one by one, 72 / 84 us by four; 256-byte rows: 103 against 105; 16 query heads to each: 61 against 68).
    const bool side_by_side = c.k_head < c.k_token && c.head_dim * type_bytes(c.dtype) % 256 != 0;
    // A row's parts then are four times as many, and so are a CTA's rows: it takes a dozen units to a CTA and as many heads to pay.
    const bool across = fours && chunk <= 8 && 4 * heads >= resident && heads * units >= 12 * (int64_t)resident && (is_8bit(c.dtype) || side_by_side);
    const int notes = (int)std::min<int64_t>(across ? heads / kWarps : heads, resident), rows = across ? kWarps * chunk : chunk;
    return {resident, 0, across, notes, rows, (notes_floats(notes) + (int64_t)resident * 2 * part_floats(rows, c.head_dim)) * 4};
}

}  // namespace
}  // namespace attn
}  // namespace pp

extern "C" pp_status_t pp_paged_attention_workspace(const pp_paged_cache_t* cache, pp_dtype_t q_type, int batch, int heads, int width,
                                                    int window, int64_t* bytes) {
    using namespace pp;
    using namespace pp::attn;
    if (!bytes) return PP_ERR_INVALID_ARG;
    *bytes = 0;
    if (const pp_status_t st = check_call(cache, q_type, batch, heads, width, window)) return st;
    if (batch == 0) return PP_OK;
    // enough for any alignment of q
    int64_t most = 0;
    for (const int q_on : {1, 16}) {
        int held[4];
        const int group = heads / cache->kv_heads;
        const Choice by = choose(*cache, q_type, q_on, group);
        if (const cudaError_t e = hold(by.form, held)) return status_of(e);
        most = std::max(most, divide(*cache, by.form, batch, width, window, by.chunk, (group + by.chunk - 1) / by.chunk, held).bytes);
    }
    *bytes = most;
    return PP_OK;
}

extern "C" pp_status_t pp_paged_attention(const pp_paged_cache_t* cache, const void* q, int64_t q_row, int64_t q_head, pp_dtype_t q_type,
                                          const int32_t* table, int64_t ld_table, int width, const int32_t* lengths, int batch, int heads,
                                          float scale, int window, void* out, float* lse, void* workspace, int64_t workspace_bytes,
                                          void* cuda_stream) {
    using namespace pp;
    using namespace pp::attn;
    if (const pp_status_t st = check_call(cache, q_type, batch, heads, width, window)) return st;
    if (!(scale > -INFINITY && scale < INFINITY)) return PP_ERR_INVALID_ARG;
    if (batch == 0) return PP_OK;
    const pp_paged_cache_t& c = *cache;
    const int tb = type_bytes(q_type);
    const int64_t most = (int64_t)1 << 56;
    if (!q || !table || !lengths || !out || q_row < 0 || q_head < 0 || q_row > most / batch || q_head > most / heads || ld_table < width || ld_table > most / batch)
        return PP_ERR_INVALID_ARG;
    if (!aligned_to(q, tb) || !aligned_to(out, tb) || !aligned_to(table, 4) || !aligned_to(lengths, 4) || !aligned_to(lse, 4) || !aligned_to(workspace, 16))
        return PP_ERR_INVALID_ARG;
    const int64_t q_span = ((batch - 1) * q_row + (heads - 1) * q_head + c.head_dim) * tb, out_span = (int64_t)batch * heads * c.head_dim * tb;
    // nothing that is written may lie on what is read, nor on one another
    const Held cached(c);
    struct Span { const void* p; int64_t bytes; };
    const Span written[] = {{out, out_span}, {lse, (int64_t)batch * heads * 4}, {workspace, workspace_bytes}};
    const Span read[] = {{q, q_span}, {table, ((int64_t)(batch - 1) * ld_table + width) * 4}, {lengths, (int64_t)batch * 4}};
    for (const Span& w : written) {
        for (const Span& r : read)
            if (spans_meet(w.p, w.bytes, r.p, r.bytes)) return PP_ERR_INVALID_ARG;
        for (const Span& other : written)
            if (&other != &w && spans_meet(w.p, w.bytes, other.p, other.bytes)) return PP_ERR_INVALID_ARG;
        if (cached.meet(w.p, w.bytes)) return PP_ERR_INVALID_ARG;
    }
    const int group = heads / c.kv_heads;
    const Choice chosen = choose(c, q_type, row_alignment(q, 1, 0, batch, q_row, heads, q_head, tb), group);
    const Form& f = chosen.form;
    const int chunk = chosen.chunk;
    int held[4];
    if (const cudaError_t e = hold(f, held)) return status_of(e);
    const int n_chunks = (group + chunk - 1) / chunk;
    const Division by = divide(c, f, batch, width, window, chunk, n_chunks, held);
    if (by.bytes && (!workspace || workspace_bytes < by.bytes)) return PP_ERR_INVALID_ARG;
    const int es = type_bytes(c.dtype);
    AttnArgs a{q, static_cast<const char*>(c.k), static_cast<const char*>(c.v), c.k_scales, c.v_scales, table, lengths, out, lse,
               static_cast<float*>(workspace), q_row, q_head, c.k_page * es, c.k_token * es, c.k_head * es, c.v_page * es, c.v_token * es,
               c.v_head * es, ld_table, Divisor((uint32_t)c.page_size), c.pages, c.page_size, batch, width * c.page_size, window, heads, c.kv_heads, group,
               chunk, n_chunks, c.head_dim, chosen.granule, q_type, c.dtype, f.inbox,
               by.notes, by.part_rows, (int64_t)batch * (by.across ? c.kv_heads / kWarps : c.kv_heads) * n_chunks <= by.grid, by.cluster,
               by.across ? kTile : kUnit, (by.across ? kTile : kUnit) % c.page_size, by.across, chosen.whole,
               c.head_dim % 4 == 0 && aligned_to(out, std::min(16, 4 * tb)), scale * kLog2e};
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    cudaError_t e = launch_pdl(f.kernel, dim3((unsigned)by.grid), dim3(kThreads), (size_t)f.smem, s, std::max(1, by.cluster), a);
    if (e == cudaSuccess && !by.cluster) {
        // few notes: a CTA for each row, then for each slice of its dimensions, if the GPU has so many
        const int rows = std::min(chunk, group) * (by.across ? kWarps : 1), room = 2 * sm_count() / a.notes;
        const int shares = std::max(1, std::min(rows, room)), slices = room >= 4 * rows ? 4 : room >= 2 * rows ? 2 : 1;
        const auto join = slices == 4 ? join_kernel<4> : slices == 2 ? join_kernel<2> : join_kernel<1>;
        e = launch_pdl(join, dim3((unsigned)a.notes, (unsigned)(shares * slices)), dim3(kJoinThreads), 0, s, 1, a, f.lift);
    }
    return status_of(e);
}
