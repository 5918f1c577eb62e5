// Matrices with 4-bit weights and group scales as a stream of units.  Shared by pp_q4.cu and pp_moe.cu.
//
//   w[m][n] = (q[m][n] - z[m][n/G]) * s[m][n/G],     q, z in 0..15
//
// A unit is 16 rows x 128 columns: 1024 bytes of codes in one array, its scales and zero points ("sets") in another, so
// that every copy of codes is whole 128-byte lines.  G is 32, 64 or a multiple of 128 (or the whole row), so a unit has 4,
// 2 or 1 sets of 16 scales (a group of 256 keeps its scale once per unit: 3 % more bytes than once per group, and no
// unit depends on another).  Units of a 16-row strip follow each other along the columns, strips follow each other.
//
// Codes: lane (g, t) = (lane / 4, lane % 4) of a warp owns rows g and g + 8 and, of every 32 columns, columns 8t .. 8t + 7.
// Its two words per 32 columns hold four columns each: byte i is column i, row g in the low half and row g + 8 in the high
// half.  Masking a word with 0x0f0f0f0f gives four codes of row g as bytes, masking it with 0xf0f0f0f0 four codes of row
// g + 8 times 16 -- both are operand registers of an integer product as they stand, and row g + 8's scale takes the 1/16.
// Zero points are kept the same way (z for the first eight rows, 16 z for the others).
#pragma once
#include "pp_decode.cuh"

namespace pp {

constexpr int kQ4UnitCols = 128;
inline __host__ __device__ int q4_sets(int group) { return group == 32 ? 4 : group == 64 ? 2 : 1; }
constexpr int kQ4CodeBytes = 1024;
inline __host__ __device__ int q4_set_bytes(int sets, bool asym) { return sets * (asym ? 48 : 32); }      // per unit
inline bool q4_group_ok(int group) { return group == 0 || group == 32 || group == 64 || (group > 0 && group % 128 == 0); }

// Rewrites `count` matrices (codes [count][rows][ceil(cols/2)], scales and zero points [count][rows][groups]) into units
// at dst (codes of [count][strips][blocks] units) and dst_sets; zeros may be null (every zero point is 8).  paired: the first and the second
// half of the rows (gate and up) share strips, eight rows of each: row g of strip s is row 8s + g of the first half, row
// 8 + g the same of the second.  In pp_q4.cu.
cudaError_t launch_q4_pack(void* dst, void* dst_sets, const void* codes, const void* scales, const void* zeros, int count, int rows, int cols,
                           int group, bool paired, cudaStream_t stream);
inline __host__ __device__ int strips_of(int rows, bool paired) { return paired ? (rows / 2 + 7) / 8 : (rows + 15) / 16; }
// Row of a matrix that row g + 8h of a strip holds, -1 where it holds none.
inline __host__ __device__ int strip_row(int rows, bool paired, int strip, int g, int h) {
    const int r = paired ? strip * 8 + g : strip * 16 + g + 8 * h;
    return r >= (paired ? rows / 2 : rows) ? -1 : paired ? r + h * (rows / 2) : r;
}

#ifdef __CUDACC__
__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
// (compiler barriers: a read of what the slot held before must not move behind the copy into it)
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async16_l1(uint32_t dst, const void* src) {         // what other warps of the SM read too
    asm volatile("cp.async.ca.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
// Shared-memory reads of the kernels' byte regions.  Plain loads, so that the compiler may order them among the products;
// the waits for asynchronous copies are compiler barriers.
template <typename T> __device__ __forceinline__ T at(const unsigned char* p) { return *reinterpret_cast<const T*>(p); }
__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm(
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

// Scales of rows g and g + 8 in a set of a unit, the second with its 1/16.
__device__ __forceinline__ float2 q4_scales(const unsigned char* slot, int set, int g, bool bf16_scales) {
    const uint32_t ss = at<uint32_t>(slot + 1024 + set * 32 + g * 4);
    float2 f;
    if (bf16_scales) f = make_float2(__uint_as_float(ss << 16), __uint_as_float(ss & 0xffff0000u));
    else f = __half22float2(*reinterpret_cast<const __half2*>(&ss));
    f.y *= 0.0625f;
    return f;
}

// tot[nt] += W_unit * X for NT tiles of 8 columns of binary16.  (word & 0x000f000f) | 0x64006400 is the pair 1024 + q of
// columns 0 and 2, adding -(1024 + z) leaves q - z exactly; four bits higher the same gives 16 (q - z), a byte further
// columns 1 and 3.  A word of eight weights costs one shift, four logic and four add instructions; products are exact,
// sums are fp32 and scaled once per set, by the row's and the column's scale.  Lane (g, t) holds in tot[nt][0..3] rows g, g,
// g + 8, g + 8 and columns 8 nt + 2t, + 1, + 0, + 1.  col_scale(nt): those two columns' scales.  load_x(nt, j): elements 8t .. 8t + 7 of the j-th 32 columns of the unit, of the lane's input column
// 8 nt + g, each four of them in the order 0, 2, 1, 3.
template <int NT, int SETS, bool ASYM, typename LoadX, typename ColScale>
__device__ __forceinline__ void q4_unit_f16(float (&tot)[NT][4], const unsigned char* slot, int lane, bool bf16_scales, LoadX load_x,
                                            ColScale col_scale) {
    const int g = lane >> 2;
    float acc[NT][4];
    uint32_t z0 = 0xE408E408u, z1 = 0xE480E480u;             // -(1024 + 8), -(1024 + 16 * 8)
    uint4 w;
#pragma unroll
    for (int j = 0; j < 4; ++j) {                            // 32 columns: two k-slices of 16
        constexpr int per_set = 4 / SETS;
        const int set = j / per_set;
        if ((j & 1) == 0) w = at<uint4>(slot + (j >> 1) * 512 + lane * 16);
        if (j % per_set == 0) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) acc[nt][0] = acc[nt][1] = acc[nt][2] = acc[nt][3] = 0.0f;
            if (ASYM) {                                      // bytes z and 16 z of rows g and g + 8
                const uint32_t zz = at<uint16_t>(slot + 1024 + SETS * 32 + set * 16 + g * 2);
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
            const float2 s = q4_scales(slot, set, g, bf16_scales);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float2 c = col_scale(nt);
                tot[nt][0] = fmaf(s.x * c.x, acc[nt][0], tot[nt][0]);
                tot[nt][1] = fmaf(s.x * c.y, acc[nt][1], tot[nt][1]);
                tot[nt][2] = fmaf(s.y * c.x, acc[nt][2], tot[nt][2]);
                tot[nt][3] = fmaf(s.y * c.y, acc[nt][3], tot[nt][3]);
            }
        }
    }
}

// ---- inputs ------------------------------------------------------------------------------------------------------
struct XIn {
    const void* x;
    const float* scales;     // 8-bit types: [tokens][scale_ld]
    int64_t ld;              // elements between tokens
    int type, scale_ld;
    int group_blocks;        // 8-bit types: blocks of 128 columns per scale, 0 = one scale per token
    int cols;
    int vec;                 // every row starts on an access of four elements and has a multiple of four
};

// Elements col .. col + 3 of a row, zeros from cols on.  VEC: rows start on an access of four elements and cols is a
// multiple of four; the load then needs no branch, and several of them stay in flight together.
template <bool VEC, typename T> __device__ __forceinline__ Pack<T, 4> load_four(const T* row, int col, int cols) {
    Pack<T, 4> v{};
    if (VEC) {
        v = *reinterpret_cast<const Pack<T, 4>*>(row + min(col, cols - 4));
        if (col >= cols) v = Pack<T, 4>{};
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (col + i < cols) v.v[i] = row[col + i];
    }
    return v;
}

// The power of two that brings a magnitude `most` to [2^13, 2^14), and its inverse; below 2^-113 the largest factor whose
// inverse is a normal number, infinities stay as they are.
__device__ __forceinline__ void f16_scale(float most, float& up, float& down) {
    uint32_t e = __float_as_uint(most) >> 23;
    e = e >= 255u ? 140u : e < 14u ? 14u : e;
    up = __uint_as_float((267u - e) << 23);
    down = __uint_as_float((e - 13u) << 23);
}

// i / n for 0 <= i < 2^20 by the reciprocal of n: an integer division takes as long as a trip to L2.
struct Divider {
    float r;
    __device__ __forceinline__ explicit Divider(int d) : r(1.0f / (float)d) {}
    __device__ __forceinline__ int div(int i) const { return (int)(((float)i + 0.5f) * r); }
};

__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t b, uint32_t sel) { return __byte_perm(a, b, sel); }

// Columns of bytes that a vector takes: an 8-bit integer is one, an e4m3 value times 2^9 a whole number of three, floats are
// fixed point of four.
template <typename T> __host__ __device__ constexpr int byte_columns() { return std::is_same_v<T, int8_t> ? 1 : sizeof(T) == 1 ? 3 : 4; }
// What column c of N stands for, in units of the last.
template <int N> __device__ __forceinline__ float byte_weight(int c) { return __int_as_float((127 + 8 * (N - 1 - c)) << 23); }

// Four whole numbers of a lane, |v| < 0.996 * 2^(8N - 1), as N words of signed bytes, the highest first.  Adding 0x80808080
// carries what a signed byte below cannot hold into the byte above; the sign bits then flip back.
template <int N> __device__ __forceinline__ void signed_bytes(const int (&v)[4], uint32_t (&w)[N]) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = ((uint32_t)v[i] + 0x80808080u) ^ 0x80808080u;
    const uint32_t a = prmt(u[0], u[1], 0x5140), b = prmt(u[2], u[3], 0x5140), c = prmt(u[0], u[1], 0x7362), d = prmt(u[2], u[3], 0x7362);
    w[N - 1] = prmt(a, b, 0x5410);
    w[N - 2] = prmt(a, b, 0x7632);
    w[N - 3] = prmt(c, d, 0x5410);
    if (N == 4) w[0] = prmt(c, d, 0x7632);
}

// A warp's block of 128 columns of one vector, four per lane: its columns' bytes and what one of them stands for (in
// `down`, of the lowest byte).  own: an 8-bit input's scale.
template <typename T> __device__ __forceinline__ void fixed_point(const Pack<T, 4>& x, float own, uint32_t (&w)[byte_columns<T>()], float& down) {
    if constexpr (std::is_same_v<T, int8_t>) {
        w[0] = *reinterpret_cast<const uint32_t*>(&x);
        down = own;
    } else if constexpr (sizeof(T) == 1) {
        int v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __float2int_rn(to_float(x.v[i]) * 512.0f);
        // NaN is the only e4m3 value that is not finite: the whole vector is not
        const bool nan = __any_sync(0xffffffffu, to_float(x.v[0]) + to_float(x.v[1]) + to_float(x.v[2]) + to_float(x.v[3]) !=
                                                     to_float(x.v[0]) + to_float(x.v[1]) + to_float(x.v[2]) + to_float(x.v[3]));
        down = nan ? __int_as_float(0x7fffffff) : own * 0x1p-9f;
        signed_bytes<3>(v, w);
    } else {
        int v[4];
        float f[4];
        uint32_t most = 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[i] = to_float(x.v[i]);
            most = max(most, __float_as_uint(f[i]) & 0x7fffffffu);        // as whole numbers: a NaN is the largest
        }
        most = __reduce_max_sync(0xffffffffu, most);
        const uint32_t e = min(max(most >> 23, 31u), 254u);                // blocks below 2^-96 keep the scale of that
        float up = __uint_as_float((284u - e) << 23);
        down = __uint_as_float((e - 30u) << 23);
        if (__uint_as_float(most) * up > 2139062016.0f) {                  // the largest float below 0x7f7f7f7f
            up *= 0.5f;
            down *= 2.0f;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __float2int_rn(f[i] * up);
        if (most >= 0x7f800000u) down = __int_as_float(0x7fffffff);        // an infinity or a NaN: so are the sums
        signed_bytes<4>(v, w);
    }
}

// The sums of a warp's N columns of bytes over each set of scales: lanes 0 .. N - 1 of a set's lanes have column `lane`'s.
template <int SETS, int N> __device__ __forceinline__ int byte_sums(const uint32_t (&w)[N], int lane) {
    constexpr int kWords = (N + 1) / 2;
    int sum[kWords];                                         // 2^16 (one column's) + (the next one's), or one alone
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
        sum[i] = __dp4a((int)w[2 * i], 0x01010101, 0);
        if (2 * i + 1 < N) sum[i] = sum[i] * 65536 + __dp4a((int)w[2 * i + 1], 0x01010101, 0);
        if (SETS == 1) {
            sum[i] = __reduce_add_sync(0xffffffffu, sum[i]);
        } else {
#pragma unroll
            for (int o = 16 / SETS; o; o >>= 1) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], o);
        }
    }
    const int c = lane & (32 / SETS - 1), s = c >= 2 && kWords > 1 ? sum[kWords - 1] : sum[0], low = (int16_t)s;
    return N == 1 || (N == 3 && c == 2) ? s : c & 1 ? low : (s - low) >> 16;
}
// Where a lane's four bytes of a block lie among its column's 128: [64 columns][lane t][8 bytes of 32 columns, 8 of the next].
__device__ __forceinline__ int byte_offset(int lane) { return (lane >> 4) * 64 + ((lane >> 1) & 3) * 16 + (lane & 8) + (lane & 1) * 4; }

__device__ __forceinline__ void mma_u8s8(int (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm(
        "mma.sync.aligned.m16n8k32.row.col.s32.u8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// tot[nt] += W_unit * X for NT tiles of 8 columns.  Lane (g, t) holds in tot[nt][0..3] rows g, g, g + 8, g + 8 and columns
// 8 nt + 2t, + 1, + 0, + 1.  load_x(nt, h): the lane's 16 bytes of its input column 8 nt + g in the h-th 64 columns of the unit;
// sums(nt, set) and col_scale(nt): of the lane's two result columns.
// The whole numbers come out of the product on top of 1.5 * 2^23: as floats they are themselves plus that, exactly, for
// magnitudes up to 2^22 (16 * 15 * 128 * 128 is less).
template <int NT, int SETS, bool ASYM, typename LoadX, typename Sums, typename ColScale>
__device__ __forceinline__ void q4_unit_i8(float (&tot)[NT][4], const unsigned char* slot, int lane, bool bf16_scales, LoadX load_x, Sums sums,
                                           ColScale col_scale) {
    constexpr int kOnTop = 0x4B400000, per_set = 4 / SETS;
    const int g = lane >> 2;
    int acc[NT][4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {                            // 64 columns: two k-slices of 32
        const uint4 w = at<uint4>(slot + h * 512 + lane * 16);
        uint4 b[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) b[nt] = load_x(nt, h);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int j = 2 * h + k, set = j / per_set;
            if (j % per_set == 0) {                          // start from -z sum d
                int z0 = -8, z1 = -128;
                if (ASYM) {
                    const uint32_t zz = at<uint16_t>(slot + 1024 + SETS * 32 + set * 16 + g * 2);
                    z0 = -(int)(zz & 255u);
                    z1 = -(int)(zz >> 8);
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const int2 d = sums(nt, set);
                    acc[nt][0] = z0 * d.x + kOnTop;
                    acc[nt][1] = z0 * d.y + kOnTop;
                    acc[nt][2] = z1 * d.x + kOnTop;
                    acc[nt][3] = z1 * d.y + kOnTop;
                }
            }
            const uint32_t w0 = k ? w.z : w.x, w1 = k ? w.w : w.y;
            const uint32_t a[4] = {w0 & 0x0f0f0f0fu, w0 & 0xf0f0f0f0u, w1 & 0x0f0f0f0fu, w1 & 0xf0f0f0f0u};
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma_u8s8(acc[nt], a, k ? b[nt].z : b[nt].x, k ? b[nt].w : b[nt].y);
            if (j % per_set == per_set - 1) {
                const float2 s = q4_scales(slot, set, g, bf16_scales);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const float2 c = col_scale(nt);
                    tot[nt][0] = fmaf(s.x * c.x, __int_as_float(acc[nt][0]) - 12582912.0f, tot[nt][0]);
                    tot[nt][1] = fmaf(s.x * c.y, __int_as_float(acc[nt][1]) - 12582912.0f, tot[nt][1]);
                    tot[nt][2] = fmaf(s.y * c.x, __int_as_float(acc[nt][2]) - 12582912.0f, tot[nt][2]);
                    tot[nt][3] = fmaf(s.y * c.y, __int_as_float(acc[nt][3]) - 12582912.0f, tot[nt][3]);
                }
            }
        }
    }
}

#endif

}  // namespace pp
