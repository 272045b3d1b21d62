// Microscaled 4-bit floating point (MXFP4, OCP microscaling formats): 32 consecutive values of a row share a power
// of two, and each is kept as one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign (E2M1).
//   e = max(floor(log2(absmax of the 32)) - 2, -127),  code = nearest E2M1 value of x 2^-e (ties to the even code, beyond 6: 6),
//   value = code 2^e; the byte of the scale is e + 127, 255 stands for "not a number".
// A block with an infinity or a NaN gets 255 and codes 0: all 32 of its values read back as NaN.
//
// Layout.  Codes: [rows][16 ceil(cols / 32)] bytes, even column in the low half, zeros past the last column: a row is
// whole 16-byte blocks, so tiles of it are TMA boxes and a block is one 16-byte access.  Scales: per 128 rows and 128
// columns one piece of 512 bytes, [32][4][4] = row % 32, row % 128 / 32, column % 128 / 32, pieces of a row tile one
// after another, an even number of them.  That is the order in which tcgen05.cp spreads them over tensor memory for a
// block-scaled product, so a product brings them in with one bulk copy and never rearranges them.
#pragma once
#include "pac_ptx.cuh"

namespace pac {

constexpr int MX_BLOCK = 32, MX_TILE = 128;
constexpr uint32_t MX_SCALE_PIECE = 512;
__host__ __device__ inline long long mx_row_bytes(int cols) { return 16LL * (((long long)cols + MX_BLOCK - 1) / MX_BLOCK); }
__host__ __device__ inline int mx_col_pieces(int cols) { return 2 * (int)(((long long)cols + 2 * MX_TILE - 1) / (2 * MX_TILE)); }
// Byte of a scale within its 512-byte piece; r = row % 128, b = block of the piece.
__host__ __device__ inline uint32_t mx_scale_at(uint32_t r, uint32_t b) { return (r & 31u) * 16u + (r >> 5) * 4u + b; }

// Eight codes of eight values times a power of two.
__device__ __forceinline__ uint32_t mx_codes8(const float* v, float f) {
    float a[8];
#pragma unroll
    for (int e = 0; e < 8; e += 2)                           // two products in one instruction
        asm("{\n .reg .b64 x, y;\n mov.b64 x, {%2, %3};\n mov.b64 y, {%4, %4};\n mul.rn.f32x2 x, x, y;\n mov.b64 {%0, %1}, x;\n}"
            : "=f"(a[e]), "=f"(a[e + 1]) : "f"(v[e]), "f"(v[e + 1]), "f"(f));
    uint32_t w;
    asm("{\n .reg .b8 b0, b1, b2, b3;\n"
        " cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n"
        " cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n"
        " mov.b32 %0, {b0, b1, b2, b3};\n}"
        : "=r"(w) : "f"(a[0]), "f"(a[1]), "f"(a[2]), "f"(a[3]), "f"(a[4]), "f"(a[5]), "f"(a[6]), "f"(a[7]));
    return w;
}
// Eight codes -> four pairs of bf16 in the order of the columns, before the scale: both bytes of |value| from a table by
// the code's low three bits (byte permutations), the sign from the code's top bit, which as a selector asks for copies of
// the table byte's top bit: ff where it is set, the byte (80) where not, so bit 6 is the sign.
__device__ __forceinline__ void mx_bf16x8(uint32_t w, uint32_t (&o)[4]) {
    uint32_t m = w & 0x77777777u, s = w;
#pragma unroll
    for (int h = 0; h < 2; ++h, m >>= 16, s >>= 16) {
        uint32_t spread;                                     // (__byte_perm would drop the selectors' top bits)
        asm("prmt.b32 %0, %1, %1, %2;" : "=r"(spread) : "r"(0x80808080u), "r"(s));
        const uint32_t sign = (spread << 1) & 0x80808080u;
        const uint32_t hi = __byte_perm(0x3f3f3f00u, 0x40404040u, m) | sign, lo = __byte_perm(0xc0800000u, 0xc0804000u, m);
        o[2 * h] = __byte_perm(lo, hi, 0x5140);
        o[2 * h + 1] = __byte_perm(lo, hi, 0x7362);
    }
}
// 2^(s - 127) as fp32, or as a pair of bf16 (2^-127 is a subnormal of both).
__device__ __forceinline__ float mx_scale_f32(uint32_t s) { return __uint_as_float(s == 0 ? 0x00400000u : s == 255 ? 0x7fffffffu : s << 23); }
__device__ __forceinline__ uint32_t mx_scale_bf16x2(uint32_t s) { return (s == 0 ? 0x0040u : s == 255 ? 0x7fffu : s << 7) * 0x10001u; }
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}

// Sixteen consecutive values as they lie in memory; `vec`: 32-byte accesses are allowed and all sixteen exist, else `have` of
// them do.  top(): the bits of the largest magnitude as fp32 (they order infinities and NaN above everything else).
template <typename T> struct MxRaw;
template <> struct MxRaw<float> {
    float v[16];
    __device__ __forceinline__ void load(const float* p, bool vec, int have) {
        if (vec && have >= 16) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
                asm volatile("ld.global.nc.L1::no_allocate.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                             : "=f"(v[8 * h]), "=f"(v[8 * h + 1]), "=f"(v[8 * h + 2]), "=f"(v[8 * h + 3]), "=f"(v[8 * h + 4]), "=f"(v[8 * h + 5]),
                               "=f"(v[8 * h + 6]), "=f"(v[8 * h + 7]) : "l"(p + 8 * h));
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e] = e < have ? p[e] : 0.f;
        }
    }
    __device__ __forceinline__ uint32_t top() const {
        uint32_t t = 0;
#pragma unroll
        for (int e = 0; e < 16; ++e) t = max(t, __float_as_uint(v[e]) & 0x7fffffffu);
        return t;
    }
    __device__ __forceinline__ void values(float (&x)[16]) const {
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = v[e];
    }
};
template <> struct MxRaw<bf16> {
    uint32_t w[8];
    __device__ __forceinline__ void load(const bf16* p, bool vec, int have) {
        if (vec && have >= 16) {
            asm volatile("ld.global.nc.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p));
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                w[e] = (2 * e < have ? (uint32_t)__bfloat16_as_ushort(p[2 * e]) : 0u) | (2 * e + 1 < have ? (uint32_t)__bfloat16_as_ushort(p[2 * e + 1]) << 16 : 0u);
        }
    }
    __device__ __forceinline__ uint32_t top() const {
        uint32_t t = 0;                                      // both halves at once
#pragma unroll
        for (int e = 0; e < 8; ++e) t = __vmaxu2(t, w[e] & 0x7fff7fffu);
        return max(t << 16, t & 0xffff0000u);
    }
    __device__ __forceinline__ void values(float (&x)[16]) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) { x[2 * e] = __uint_as_float(w[e] << 16); x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u); }
    }
};

// n / d for d >= 1: a multiplication by m = ceil(2^(31 + s) / d), 2^s >= d > 2^(s-1), where n < 2^31 (m < 2^32, and what m is too
// large by adds less than n / 2^31 / d to the quotient); a 64-bit division otherwise.  (The codec spent a third of its
// instructions on the latter.)
struct MxDiv {
    long long d;
    uint32_t m, s;                                          // m == 0: d is 1
    bool small;
    MxDiv(long long d_, long long most) : d(d_), m(0), s(1), small(most < (1LL << 31) && d_ < (1LL << 31)) {
        while ((1LL << s) < d) ++s;
        if (small && d > 1) m = (uint32_t)(((1ULL << (31 + s)) + (unsigned long long)d - 1) / (unsigned long long)d);
    }
    __device__ __forceinline__ long long div(long long n) const {
        if (!small) return n / d;
        return m ? (long long)(__umulhi((uint32_t)n, m) >> (s - 1)) : n;
    }
};

// A warp takes four rows and 256 columns (two pieces of scales) at a time: eight lanes to a row, sixteen values to a lane
// and piece, two lanes to a block.  The rows and pieces that only fill up a tile are walked too: their scales are written
// as 0, so that a product may read whole pieces.  Bound by HBM (4.53 or 2.53 bytes per value).
template <typename T>
__global__ void __launch_bounds__(256) quantize_mxfp_kernel(const T* __restrict__ x, long long rows, int cols, long long ldx, bool vec,
                                                            unsigned char* __restrict__ codes, unsigned char* __restrict__ scales, const MxDiv by_pairs) {
    const int lane = threadIdx.x & 31, in_row = lane & 7;
    const int pieces = mx_col_pieces(cols);
    const long long row_bytes = mx_row_bytes(cols);
    const long long groups = (rows + MX_TILE - 1) / MX_TILE * (MX_TILE / 4), items = groups * (pieces / 2);
    const long long warps = ((long long)gridDim.x * blockDim.x) >> 5;
    for (long long it = ((long long)blockIdx.x * blockDim.x + threadIdx.x) >> 5; it < items; it += warps) {
        const long long g = by_pairs.div(it);
        const int cp = 2 * (int)(it - g * (pieces / 2));
        const long long row = g * 4 + (lane >> 3);
        MxRaw<T> raw[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int c0 = (cp + h) * MX_TILE + in_row * 16;
            raw[h].load(x + row * ldx + c0, vec, row < rows ? cols - c0 : 0);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t top = raw[h].top();
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            const uint32_t ex = top >> 23;
            const bool finite = ex < 255u;
            const uint32_t s = finite ? (ex > 2u ? ex - 2u : 0u) : 255u;
            const float f = finite ? __uint_as_float((254u - s) << 23) : 0.f;      // 2^(127 - s); s <= 252
            const int c0 = (cp + h) * MX_TILE + in_row * 16;
            if (row < rows && (c0 & ~31) < cols) {
                uint2 w = make_uint2(0u, 0u);
                float v[16];
                raw[h].values(v);
                if (finite) w = make_uint2(mx_codes8(v, f), mx_codes8(v + 8, f));
                *reinterpret_cast<uint2*>(codes + row * row_bytes + (c0 >> 1)) = w;
            }
            // the four scales of a row and piece as one word
            uint32_t word = (in_row & 1) ? 0u : s << (4 * in_row);
            word |= __shfl_xor_sync(0xffffffffu, word, 2);
            word |= __shfl_xor_sync(0xffffffffu, word, 4);
            if (in_row == 0) {
                unsigned char* piece = scales + ((row / MX_TILE) * pieces + cp + h) * (long long)MX_SCALE_PIECE;
                *reinterpret_cast<uint32_t*>(piece + mx_scale_at((uint32_t)(row % MX_TILE), 0u)) = word;
            }
        }
    }
}

// Sixteen values to a lane, as above; rows begin on 32-byte boundaries.  Bound by HBM.
template <typename T>
__global__ void __launch_bounds__(256) dequantize_mxfp_kernel(const unsigned char* __restrict__ codes, const unsigned char* __restrict__ scales,
                                                              long long rows, int cols, T* __restrict__ out, long long ldo, const MxDiv by_row) {
    const int pieces = mx_col_pieces(cols);
    const long long row_bytes = mx_row_bytes(cols);
    const long long per_row = row_bytes >> 3, items = rows * per_row;
    for (long long it = (long long)blockIdx.x * blockDim.x + threadIdx.x; it < items; it += (long long)gridDim.x * blockDim.x) {
        const long long row = by_row.div(it);
        const int at = (int)(it - row * per_row), c0 = at * 16;
        const uint2 w = *reinterpret_cast<const uint2*>(codes + it * 8);
        const uint32_t s = scales[((row / MX_TILE) * pieces + c0 / MX_TILE) * (long long)MX_SCALE_PIECE + mx_scale_at((uint32_t)(row % MX_TILE), (uint32_t)(c0 % MX_TILE) / MX_BLOCK)];
        uint32_t o[2][4];
        mx_bf16x8(w.x, o[0]);
        mx_bf16x8(w.y, o[1]);
        if constexpr (sizeof(T) == 2) {                      // a value times its power of two is a bf16 exactly
            const uint32_t f = mx_scale_bf16x2(s);
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e >> 2][e & 3] = mul_bf16x2(o[e >> 2][e & 3], f);
        }
        float v[16];
        if constexpr (sizeof(T) == 4) {
            const float f = mx_scale_f32(s);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[2 * e] = __uint_as_float(o[e >> 2][e & 3] << 16) * f;
                v[2 * e + 1] = __uint_as_float(o[e >> 2][e & 3] & 0xffff0000u) * f;
            }
        }
        T* dst = out + row * ldo + c0;
        if (c0 + 16 <= cols) {
            if constexpr (sizeof(T) == 4) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    st_global_32(dst + 8 * h, make_uint4(__float_as_uint(v[8 * h]), __float_as_uint(v[8 * h + 1]), __float_as_uint(v[8 * h + 2]), __float_as_uint(v[8 * h + 3])),
                                 make_uint4(__float_as_uint(v[8 * h + 4]), __float_as_uint(v[8 * h + 5]), __float_as_uint(v[8 * h + 6]), __float_as_uint(v[8 * h + 7])));
            } else {
                st_global_32(dst, make_uint4(o[0][0], o[0][1], o[0][2], o[0][3]), make_uint4(o[1][0], o[1][1], o[1][2], o[1][3]));
            }
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (c0 + e < cols) {
                    if constexpr (sizeof(T) == 4) dst[e] = v[e];
                    else dst[e] = __ushort_as_bfloat16((unsigned short)(o[e >> 3][(e >> 1) & 3] >> (16 * (e & 1))));
                }
        }
    }
}
// Rows that do not begin on 32-byte boundaries: two values to a lane, so that a warp's stores are neighbours (sixteen to a lane
// and element by element, 8192 x 770 took 38 us).
template <typename T>
__global__ void __launch_bounds__(256) dequantize_mxfp_any_kernel(const unsigned char* __restrict__ codes, const unsigned char* __restrict__ scales,
                                                                  long long rows, int cols, T* __restrict__ out, long long ldo, const MxDiv by_row) {
    const int pieces = mx_col_pieces(cols);
    const long long row_bytes = mx_row_bytes(cols), items = rows * row_bytes;
    for (long long it = (long long)blockIdx.x * blockDim.x + threadIdx.x; it < items; it += (long long)gridDim.x * blockDim.x) {
        const long long row = by_row.div(it);
        const int c0 = 2 * (int)(it - row * row_bytes);
        const uint32_t w = codes[it];
        const float f = mx_scale_f32(scales[((row / MX_TILE) * pieces + c0 / MX_TILE) * (long long)MX_SCALE_PIECE + mx_scale_at((uint32_t)(row % MX_TILE), (uint32_t)(c0 % MX_TILE) / MX_BLOCK)]);
        uint32_t o[4];
        mx_bf16x8(w, o);
        T* dst = out + row * ldo + c0;
#pragma unroll
        for (int e = 0; e < 2; ++e)
            if (c0 + e < cols) {
                const float v = __uint_as_float(e ? o[0] & 0xffff0000u : o[0] << 16) * f;
                if constexpr (sizeof(T) == 4) dst[e] = v;
                else dst[e] = __float2bfloat16(v);
            }
    }
}

}  // namespace pac
