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

// Sixteen codes of sixteen values times a power of two.
__device__ __forceinline__ uint32_t mx_codes8(const float* v, float f) {
    uint32_t w;
    asm("{\n .reg .b8 b0, b1, b2, b3;\n"
        " cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n"
        " cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n"
        " mov.b32 %0, {b0, b1, b2, b3};\n}"
        : "=r"(w) : "f"(v[0] * f), "f"(v[1] * f), "f"(v[2] * f), "f"(v[3] * f), "f"(v[4] * f), "f"(v[5] * f), "f"(v[6] * f), "f"(v[7] * f));
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

// Sixteen consecutive values; `vec`: 32-byte accesses are allowed and all sixteen exist.  `have` of them exist otherwise.
__device__ __forceinline__ void mx_load16(const float* p, bool vec, int have, float (&v)[16]) {
    if (vec) {
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
__device__ __forceinline__ void mx_load16(const bf16* p, bool vec, int have, float (&v)[16]) {
    if (vec) {
        uint32_t u[8];
        asm volatile("ld.global.nc.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]) : "l"(p));
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[2 * e] = __uint_as_float(u[e] << 16);
            v[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = e < have ? __bfloat162float(p[e]) : 0.f;
    }
}

// A warp takes four rows and 256 columns (two pieces of scales) at a time: eight lanes to a row, sixteen values to a lane
// and piece, two lanes to a block.  The rows and pieces that only fill up a tile are walked too: their scales are written
// as 0, so that a product may read whole pieces.  Bound by HBM (4.53 or 2.53 bytes per value).
template <typename T>
__global__ void __launch_bounds__(256) quantize_mxfp_kernel(const T* __restrict__ x, long long rows, int cols, long long ldx, bool vec,
                                                            unsigned char* __restrict__ codes, unsigned char* __restrict__ scales) {
    const int lane = threadIdx.x & 31, in_row = lane & 7;
    const int pieces = mx_col_pieces(cols);
    const long long row_bytes = mx_row_bytes(cols);
    const long long groups = (rows + MX_TILE - 1) / MX_TILE * (MX_TILE / 4), items = groups * (pieces / 2);
    const long long warps = ((long long)gridDim.x * blockDim.x) >> 5;
    for (long long it = ((long long)blockIdx.x * blockDim.x + threadIdx.x) >> 5; it < items; it += warps) {
        const long long g = it / (pieces / 2);
        const int cp = 2 * (int)(it - g * (pieces / 2));
        const long long row = g * 4 + (lane >> 3);
        float v[2][16];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int c0 = (cp + h) * MX_TILE + in_row * 16;
            const int have = row < rows ? cols - c0 : 0;
            if (have > 0) mx_load16(x + row * ldx + c0, vec && have >= 16, have, v[h]);
            else {
#pragma unroll
                for (int e = 0; e < 16; ++e) v[h][e] = 0.f;
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            // the largest magnitude as bits: orders infinities and NaN above everything else
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < 16; ++e) top = max(top, __float_as_uint(v[h][e]) & 0x7fffffffu);
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            const uint32_t ex = top >> 23;
            const bool finite = ex < 255u;
            const uint32_t s = finite ? (ex > 2u ? ex - 2u : 0u) : 255u;
            const float f = finite ? __uint_as_float((254u - s) << 23) : 0.f;      // 2^(127 - s); s <= 252
            const int c0 = (cp + h) * MX_TILE + in_row * 16;
            if (row < rows && (c0 & ~31) < cols) {
                uint2 w = make_uint2(0u, 0u);
                if (finite) w = make_uint2(mx_codes8(&v[h][0], f), mx_codes8(&v[h][8], f));
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

// Sixteen values to a lane, as above.  Bound by HBM.
template <typename T>
__global__ void __launch_bounds__(256) dequantize_mxfp_kernel(const unsigned char* __restrict__ codes, const unsigned char* __restrict__ scales,
                                                              long long rows, int cols, T* __restrict__ out, long long ldo, bool vec) {
    const int pieces = mx_col_pieces(cols);
    const long long row_bytes = mx_row_bytes(cols);
    const long long per_row = row_bytes >> 3, items = rows * per_row;
    for (long long it = (long long)blockIdx.x * blockDim.x + threadIdx.x; it < items; it += (long long)gridDim.x * blockDim.x) {
        const long long row = it / per_row;
        const int at = (int)(it - row * per_row), c0 = at * 16;
        const uint2 w = *reinterpret_cast<const uint2*>(codes + it * 8);
        const uint32_t s = scales[((row / MX_TILE) * pieces + c0 / MX_TILE) * (long long)MX_SCALE_PIECE + mx_scale_at((uint32_t)(row % MX_TILE), (uint32_t)(c0 % MX_TILE) / MX_BLOCK)];
        uint32_t o[2][4];
        mx_bf16x8(w.x, o[0]);
        mx_bf16x8(w.y, o[1]);
        const float f = mx_scale_f32(s);
        float v[16];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[2 * e] = __uint_as_float(o[e >> 2][e & 3] << 16) * f;
            v[2 * e + 1] = __uint_as_float(o[e >> 2][e & 3] & 0xffff0000u) * f;
        }
        T* dst = out + row * ldo + c0;
        if (vec && c0 + 16 <= cols) {
            if constexpr (sizeof(T) == 4) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    st_global_32(dst + 8 * h, make_uint4(__float_as_uint(v[8 * h]), __float_as_uint(v[8 * h + 1]), __float_as_uint(v[8 * h + 2]), __float_as_uint(v[8 * h + 3])),
                                 make_uint4(__float_as_uint(v[8 * h + 4]), __float_as_uint(v[8 * h + 5]), __float_as_uint(v[8 * h + 6]), __float_as_uint(v[8 * h + 7])));
            } else {
                uint32_t u[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) u[e] = bf16_pair(v[2 * e], v[2 * e + 1]);
                st_global_32(dst, make_uint4(u[0], u[1], u[2], u[3]), make_uint4(u[4], u[5], u[6], u[7]));
            }
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (c0 + e < cols) {
                    if constexpr (sizeof(T) == 4) dst[e] = v[e];
                    else dst[e] = __float2bfloat16(v[e]);
                }
        }
    }
}

}  // namespace pac
