// Matrices with 4-bit weights and group scales as a stream of units, and the product of one unit with the columns
// of a staged input.  Shared by pp_q4.cu and pp_moe.cu.
//
//   w[m][n] = (q[m][n] - z[m][n/G]) * s[m][n/G],     q, z in 0..15
//
// A unit is 16 rows x 128 columns: 1024 bytes of codes, then the unit's scales and zero points.  G is 32, 64 or a
// multiple of 128 (or the whole row), so a unit holds 4, 2 or 1 sets of 16 scales (a group of 256 keeps its scale
// once per unit: 3 % more bytes than once per group, and no unit depends on another).  Units of a 16-row strip
// follow each other along the columns, strips follow each other.
//
// The codes go through the 16x8x16 tensor-core instruction as exact small integers in binary16:
// (word & 0x000f000f) | 0x64006400 is the pair 1024 + q, and subtracting 1024 + z leaves q - z.  Where the nibble
// sits four bits higher the same two instructions give 1024 + 16q and 16(q - z); those are always the rows 8..15 of
// the unit, whose scale takes the 1/16.  So a word of eight weights costs one shift, four logic and four add
// instructions, products are exact, and sums are held in fp32 and scaled once per set.
// (Leaving out the subtraction and correcting by z * sum(x) would save four of the nine, but sums of q x without
// the offset lose up to four more bits when x has a mean, as it does behind a ReLU.)
#pragma once
#include "pp_decode.cuh"

namespace pp {

constexpr int kQ4UnitCols = 128;
inline __host__ __device__ int q4_sets(int group) { return group == 32 ? 4 : group == 64 ? 2 : 1; }
inline __host__ __device__ int q4_unit_bytes(int sets, bool asym) { return 1024 + sets * (asym ? 48 : 32); }
inline bool q4_group_ok(int group) { return group == 0 || group == 32 || group == 64 || (group > 0 && group % 128 == 0); }

// Rewrites `count` matrices (codes [count][rows][ceil(cols/2)], scales and zero points [count][rows][groups]) into units
// at dst ([count][strips][blocks] units); zeros may be null (every zero point is 8).  paired: the first and the second
// half of the rows (gate and up) share strips, eight rows of each: row g of strip s is row 8s + g of the first half, row
// 8 + g the same of the second.  In pp_q4.cu.
cudaError_t launch_q4_pack(void* dst, const void* codes, const void* scales, const void* zeros, int count, int rows, int cols,
                           int group, bool paired, cudaStream_t stream);
inline __host__ __device__ int strips_of(int rows, bool paired) { return paired ? (rows / 2 + 7) / 8 : (rows + 15) / 16; }
// Row of a matrix that row g + 8h of a strip holds, -1 where it holds none.
inline __host__ __device__ int strip_row(int rows, bool paired, int strip, int g, int h) {
    const int r = paired ? strip * 8 + g : strip * 16 + g + 8 * h;
    return r >= (paired ? rows / 2 : rows) ? -1 : paired ? r + h * (rows / 2) : r;
}

#ifdef __CUDACC__
__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src));
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ uint4 lds128(uint32_t a) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
    return v;
}
__device__ __forceinline__ float2 lds_f2(uint32_t a) {
    float2 v;
    asm volatile("ld.shared.v2.f32 {%0,%1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(a));
    return v;
}
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a));
    return v;
}
__device__ __forceinline__ uint32_t lds16(uint32_t a) {
    uint16_t v;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(a));
    return v;
}
__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t hadd2_bits(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("add.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
template <uint32_t MASK> __device__ __forceinline__ uint32_t code_pair(uint32_t w) {   // (w & MASK) | 0x64006400
    uint32_t d;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(d) : "r"(w), "n"(MASK), "n"(0x64006400));
    return d;
}

// One lane's 16 bytes per chunk of a unit: asynchronous copies of `bytes` (a multiple of 16) by a warp.
__device__ __forceinline__ void q4_fetch(uint32_t slot, const unsigned char* unit, int lane, int extra16) {
    cp_async16(slot + lane * 16, unit + lane * 16);
    cp_async16(slot + 512 + lane * 16, unit + 512 + lane * 16);
    if (lane < extra16) cp_async16(slot + 1024 + lane * 16, unit + 1024 + lane * 16);
}

// tot[nt] += W_unit * X for NT tiles of 8 columns.  Lane (g, t) = (lane / 4, lane % 4) holds in tot[nt][0..3] rows g, g,
// g + 8, g + 8 and columns 8 nt + 2t, + 1, + 0, + 1.  load_x(nt, j): elements 8t .. 8t + 7 of the j-th 32 columns of the
// unit, of the lane's input column 8 nt + g.  col_scale(nt): the input's own scales for this unit and the lane's two
// result columns.
template <int NT, int SETS, bool ASYM, typename LoadX, typename ColScale>
__device__ __forceinline__ void q4_unit(float (&tot)[NT][4], uint32_t slot, int lane, bool bf16_scales, LoadX load_x, ColScale col_scale) {
    const int g = lane >> 2;
    float acc[NT][4];
    uint32_t z0 = 0xE408E408u, z1 = 0xE480E480u;             // -(1024 + 8), -(1024 + 16 * 8)
    uint4 w;
#pragma unroll
    for (int j = 0; j < 4; ++j) {                            // 32 columns: two k-slices of 16
        constexpr int per_set = 4 / SETS;
        const int set = j / per_set;
        if ((j & 1) == 0) w = lds128(slot + (j >> 1) * 512 + lane * 16);
        if (j % per_set == 0) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) acc[nt][0] = acc[nt][1] = acc[nt][2] = acc[nt][3] = 0.0f;
            if (ASYM) {                                      // bytes z and 16 z of rows g and g + 8
                const uint32_t zz = lds16(slot + 1024 + SETS * 32 + set * 16 + g * 2);
                z0 = __byte_perm(zz, 0x000000E4u, 0x4040);
                z1 = __byte_perm(zz, 0x000000E4u, 0x4141);
            }
        }
        const uint32_t w0 = (j & 1) ? w.z : w.x, w1 = (j & 1) ? w.w : w.y;
        uint32_t a[4], b[4];
        a[0] = hadd2_bits(code_pair<0x000f000f>(w0), z0);
        a[1] = hadd2_bits(code_pair<0x00f000f0>(w0), z1);
        a[2] = hadd2_bits(code_pair<0x000f000f>(w0 >> 8), z0);
        a[3] = hadd2_bits(code_pair<0x00f000f0>(w0 >> 8), z1);
        b[0] = hadd2_bits(code_pair<0x000f000f>(w1), z0);
        b[1] = hadd2_bits(code_pair<0x00f000f0>(w1), z1);
        b[2] = hadd2_bits(code_pair<0x000f000f>(w1 >> 8), z0);
        b[3] = hadd2_bits(code_pair<0x00f000f0>(w1 >> 8), z1);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const uint4 x = load_x(nt, j);
            mma_f16(acc[nt], a, x.x, x.y);
            mma_f16(acc[nt], b, x.z, x.w);
        }
        if (j % per_set == per_set - 1) {
            const uint32_t ss = lds32(slot + 1024 + set * 32 + g * 4);
            float s0, s1;
            if (bf16_scales) {
                s0 = __uint_as_float(ss << 16);
                s1 = __uint_as_float(ss & 0xffff0000u);
            } else {
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&ss));
                s0 = f.x;
                s1 = f.y;
            }
            s1 *= 0.0625f;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float2 c = col_scale(nt);
                tot[nt][0] = fmaf(s0 * c.x, acc[nt][0], tot[nt][0]);
                tot[nt][1] = fmaf(s0 * c.y, acc[nt][1], tot[nt][1]);
                tot[nt][2] = fmaf(s1 * c.x, acc[nt][2], tot[nt][2]);
                tot[nt][3] = fmaf(s1 * c.y, acc[nt][3], tot[nt][3]);
            }
        }
    }
}

// ---- staging of the input ------------------------------------------------------------------------------------
// A token's row becomes one or two columns of binary16 with an fp32 scale per 128 columns, so that columns times scale
// is the input: f16 and the 8-bit types are themselves (their own scale); bf16 is multiplied by the power of two that
// brings the block's largest magnitude to [2^13, 2^14) -- exact but for elements 2^-30 of that magnitude and less,
// which fp32 sums could not see either; f32 takes a second column for what the first one's 11 bits leave over
// (together as exact as fp32 rounding).
__host__ __device__ __forceinline__ int columns_per_token(int xtype) { return xtype == PP_F32 ? 2 : 1; }

struct XIn {
    const void* x;
    const float* scales;     // 8-bit types: [tokens][scale_ld]
    int64_t ld;              // elements between tokens
    int type, scale_ld;
    int group_blocks;        // 8-bit types: blocks of 128 columns per scale, 0 = one scale per token
    int cols;
    int vec;                 // every row starts on an access of four elements
};

__device__ __forceinline__ void load_four(float (&v)[4], const XIn& in, int64_t at, int col) {
    const bool whole = in.vec && col + 4 <= in.cols;
    v[0] = v[1] = v[2] = v[3] = 0.0f;
    switch (in.type) {
        case PP_F32: {
            const float* p = static_cast<const float*>(in.x) + at + col;
            if (whole) load_vec(v, p);
            else
                for (int i = 0; i < 4; ++i) if (col + i < in.cols) v[i] = p[i];
            break;
        }
        case PP_F16: {
            const __half* p = static_cast<const __half*>(in.x) + at + col;
            if (whole) load_vec(v, p);
            else
                for (int i = 0; i < 4; ++i) if (col + i < in.cols) v[i] = to_float(p[i]);
            break;
        }
        case PP_BF16: {
            const __nv_bfloat16* p = static_cast<const __nv_bfloat16*>(in.x) + at + col;
            if (whole) load_vec(v, p);
            else
                for (int i = 0; i < 4; ++i) if (col + i < in.cols) v[i] = to_float(p[i]);
            break;
        }
        case PP_I8: {
            const int8_t* p = static_cast<const int8_t*>(in.x) + at + col;
            if (whole) load_vec(v, p);
            else
                for (int i = 0; i < 4; ++i) if (col + i < in.cols) v[i] = to_float(p[i]);
            break;
        }
        default: {
            const __nv_fp8_e4m3* p = static_cast<const __nv_fp8_e4m3*>(in.x) + at + col;
            if (whole) load_vec(v, p);
            else
                for (int i = 0; i < 4; ++i) if (col + i < in.cols) v[i] = to_float(p[i]);
            break;
        }
    }
}

// The power of two that brings a magnitude `most` (a block's largest) to [2^13, 2^14), and its inverse; blocks below
// 2^-113 take the largest factor whose inverse is a normal number, one with an infinity in it keeps its values.
__device__ __forceinline__ void block_scale(float most, float& up, float& down) {
    uint32_t e = __float_as_uint(most) >> 23;
    e = e >= 255u ? 140u : e < 14u ? 14u : e;
    up = __uint_as_float((267u - e) << 23);
    down = __uint_as_float((e - 13u) << 23);
}

__device__ __forceinline__ uint2 four_halves(const float (&v)[4]) {
    const __half2 lo = __floats2half2_rn(v[0], v[1]), hi = __floats2half2_rn(v[2], v[3]);
    return make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
}

// A warp converts one token's block of 128 columns (four per lane).  dst: halves of the token's first column in the
// block's first 32 columns; step: halves to the next 32 columns (the second column of an f32 token is 32 halves on).
__device__ __forceinline__ float stage_block(const float (&v)[4], const XIn& in, int token, int block, __half* dst, int step) {
    const int lane = threadIdx.x & 31;
    uint2* at = reinterpret_cast<uint2*>(dst + (lane >> 3) * step + (lane & 7) * 4);
    if (in.type == PP_F16 || in.type == PP_I8 || in.type == PP_E4M3) {
        *at = four_halves(v);
        if (in.type == PP_F16) return 1.0f;
        return in.scales[(int64_t)token * in.scale_ld + (in.group_blocks ? block / in.group_blocks : 0)];
    }
    float most = fmaxf(fmaxf(fabsf(v[0]), fabsf(v[1])), fmaxf(fabsf(v[2]), fabsf(v[3])));
#pragma unroll
    for (int o = 16; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
    float up, down, s[4];
    block_scale(most, up, down);
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = v[i] * up;
    const uint2 hi = four_halves(s);
    *at = hi;
    if (in.type == PP_F32) {
        const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&hi.x)), b = __half22float2(*reinterpret_cast<const __half2*>(&hi.y));
        const float rest[4] = {s[0] - a.x, s[1] - a.y, s[2] - b.x, s[3] - b.y};
        at[8] = four_halves(rest);                           // 32 halves further on
    }
    return down;
}
#endif

}  // namespace pp
