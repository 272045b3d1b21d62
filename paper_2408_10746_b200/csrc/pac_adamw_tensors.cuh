// One AdamW step over a list of tensors in one launch, moments in fp32 or in 8 bits.
//
//   m = b1 m + (1-b1) g;  v = b2 v + ((1-b2) g) g;  p = (p - lr wd p) - lr (m / bc1) / (sqrt(v / bc2) + eps)
//
// 8 bits: m and sqrt(v) are kept as float8 (E4M3) times an fp32 constant per 256 elements, absmax / 448.  The root halves
// the range of exponents that has to fit.  With beta2 = 0.999 a step moves v by a thousandth and neighbouring codes are
// an eighth apart, so rounding to the nearest would hold v where it is for ever; codes are rounded up or down by 16
// random bits instead (up with the probability of the remainder), which keeps the averages unbiased.  The bits are a hash
// of (seed, step, tensor, element): the same call gives the same codes.  A root that is not 0 never becomes 0, so a
// moment never meets a denominator of eps alone.  A block with a gradient that is not finite gets the constant NaN.
//
// The step reads and writes every element once: 28 bytes (fp32 everywhere), 16 (moments in 8 bits), 10 (bf16 parameters
// and gradients on top).  A warp takes 256 elements, eight per lane, so the block's maximum is five shuffles and the
// moments never leave its registers between decoding and encoding.  The list is an argument of the kernel (constant
// memory): nothing to copy, nothing to keep alive after the call, capturable.
#pragma once
#include "pac_ptx.cuh"
#include "pac_adamw.cuh"

namespace pac {

constexpr int AT_BLOCK = 256, AT_SMALL = 48, AT_LARGE = 480;
struct AtTensor {
    void* p; const void* g; void* m; void* v;
    float* m_scale; float* v_scale;
    long long n;
    uint32_t first_block;       // blocks of 256 elements ahead of this tensor's
    uint32_t flags;             // see AT_*
};
constexpr uint32_t AT_P16 = 1u, AT_G16 = 2u, AT_DECAY = 4u, AT_VEC = 8u;
template <int CAP>
struct AtList { AtTensor t[CAP]; };
struct AtStep {
    int count, first_tensor;    // tensors of this launch; the first one's place in the caller's list (names its random bits)
    uint32_t blocks;
    pac_adamw hp;
    float bc1, bc2, grad_scale;
    uint32_t seed, step;
    const long long* dev_step;  // when given: the number of the step, in place of step, bc1, bc2
};

// A bijection of 32 bits whose every output bit depends on every input bit: two multiplications between xor-shifts.
__host__ __device__ __forceinline__ uint32_t at_mix(uint32_t x) {
    x ^= x >> 16; x *= 0x85EBCA6Bu;
    x ^= x >> 13; x *= 0xC2B2AE35u;
    return x ^ (x >> 16);
}

// Eight elements e(j) of a block: consecutive per lane (vec) or one of each 32 (any alignment).
__device__ __forceinline__ int at_elem(bool vec, int lane, int j) { return vec ? lane * 8 + j : j * 32 + lane; }

__device__ __forceinline__ void at_load(const void* base, long long i0, bool is16, bool vec, int lane, int len, float (&x)[8]) {
    if (vec && len == AT_BLOCK) {
        if (is16) {
            const uint4 u = *reinterpret_cast<const uint4*>(static_cast<const bf16*>(base) + i0 + lane * 8);
            const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) { x[2 * j] = __uint_as_float(w[j] << 16); x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u); }
        } else {
            asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7])
                         : "l"(static_cast<const float*>(base) + i0 + lane * 8));
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int e = at_elem(vec, lane, j);
            x[j] = e >= len ? 0.f : is16 ? __bfloat162float(static_cast<const bf16*>(base)[i0 + e]) : static_cast<const float*>(base)[i0 + e];
        }
    }
}
__device__ __forceinline__ void at_store(void* base, long long i0, bool is16, bool vec, int lane, int len, const float (&x)[8]) {
    if (vec && len == AT_BLOCK) {
        if (is16) {
            *reinterpret_cast<uint4*>(static_cast<bf16*>(base) + i0 + lane * 8) =
                make_uint4(bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7]));
        } else {
            st_global_32(static_cast<float*>(base) + i0 + lane * 8,
                         make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])),
                         make_uint4(__float_as_uint(x[4]), __float_as_uint(x[5]), __float_as_uint(x[6]), __float_as_uint(x[7])));
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int e = at_elem(vec, lane, j);
            if (e < len) {
                if (is16) static_cast<bf16*>(base)[i0 + e] = __float2bfloat16(x[j]);
                else static_cast<float*>(base)[i0 + e] = x[j];
            }
        }
    }
}
__device__ __forceinline__ uint2 at_load_codes(const void* base, long long i0, bool vec, int lane, int len) {
    const unsigned char* p = static_cast<const unsigned char*>(base) + i0;
    if (vec && len == AT_BLOCK) return *reinterpret_cast<const uint2*>(p + lane * 8);
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int e = at_elem(vec, lane, j);
        if (e < len) w[j >> 2] |= (uint32_t)p[e] << (8 * (j & 3));
    }
    return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ void at_store_codes(void* base, long long i0, bool vec, int lane, int len, uint2 c) {
    unsigned char* p = static_cast<unsigned char*>(base) + i0;
    if (vec && len == AT_BLOCK) { *reinterpret_cast<uint2*>(p + lane * 8) = c; return; }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int e = at_elem(vec, lane, j);
        if (e < len) p[e] = (unsigned char)((j < 4 ? c.x : c.y) >> (8 * (j & 3)));
    }
}
// Eight E4M3 codes -> fp32 (exact).
__device__ __forceinline__ void at_decode(uint2 c, float (&x)[8]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t w = (j < 2 ? c.x : c.y) >> (16 * (j & 1));
        uint32_t h;
        asm("{\n .reg .b16 t;\n cvt.u16.u32 t, %1;\n cvt.rn.f16x2.e4m3x2 %0, t;\n}" : "=r"(h) : "r"(w & 0xffffu));
        asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %2;\n cvt.f32.f16 %0, a;\n cvt.f32.f16 %1, b;\n}" : "=f"(x[2 * j]), "=f"(x[2 * j + 1]) : "r"(h));
    }
}
// Constant of a block and the factor into E4M3's range, from the bits of its largest magnitude.
__device__ __forceinline__ void at_constant(uint32_t top_bits, float& scale, float& f) {
    const float top = __uint_as_float(top_bits);
    if (top_bits >= 0x7f800000u) { scale = __uint_as_float(0x7fffffffu); f = 0.f; }
    else if (top < 7.888609052210118e-31f) { scale = 0.f; f = 0.f; }            // 2^-100: 448 / top would overflow further down
    else { scale = __fdiv_rn(top, 448.f); f = __fdiv_rn(448.f, top); }
}
// E4M3 code of a magnitude r in [0, 448], rounded up with the probability of what is cut off; `bits`: 16 random bits.
__device__ __forceinline__ uint32_t at_code(float r, uint32_t bits) {
    const uint32_t add = bits << 4;
    // normal codes: three bits of the fraction stay; below 2^-6 the steps are 2^-9
    if (r < 0.015625f) return ((uint32_t)(r * 536870912.f) + add) >> 20;
    return ((__float_as_uint(r) + add) >> 20) - 960u;
}

template <int BITS, int CAP>
__global__ void __launch_bounds__(256) adamw_tensors_kernel(const __grid_constant__ AtList<CAP> list, AtStep s) {
    const int lane = threadIdx.x & 31;
    __shared__ float bc_sh[2];
    uint32_t step = s.step;
    float bc1 = s.bc1, bc2 = s.bc2;
    if (s.dev_step) {
        const long long st = *s.dev_step;
        step = (uint32_t)st;
        if (threadIdx.x < 2) bc_sh[threadIdx.x] = (float)(1.0 - pow((double)(threadIdx.x ? s.hp.beta2 : s.hp.beta1), (double)st));
        __syncthreads();
        bc1 = bc_sh[0]; bc2 = bc_sh[1];
    }
    const float rbc1 = __fdiv_rn(1.f, bc1), rroot2 = __fdiv_rn(1.f, __fsqrt_rn(bc2));
    const float omb1 = __fsub_rn(1.f, s.hp.beta1), omb2 = __fsub_rn(1.f, s.hp.beta2), lrwd = __fmul_rn(s.hp.lr, s.hp.weight_decay);
    const uint32_t step_key = BITS == 8 ? at_mix(s.seed + 0x9E3779B9u * step) : 0u;
    const uint32_t warps = (gridDim.x * blockDim.x) >> 5;
    for (uint32_t b = (blockIdx.x * blockDim.x + threadIdx.x) >> 5; b < s.blocks; b += warps) {
        int lo = 0, hi = s.count - 1;                       // the last tensor that begins at or before block b
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (list.t[mid].first_block <= b) lo = mid; else hi = mid - 1;
        }
        const AtTensor& t = list.t[lo];
        const uint32_t tb = b - t.first_block, flags = t.flags;
        const long long i0 = (long long)tb * AT_BLOCK;
        const int len = (int)min((long long)AT_BLOCK, t.n - i0);
        const bool vec = flags & AT_VEC;
        float p[8], g[8], m[8], v[8];
        at_load(t.g, i0, flags & AT_G16, vec, lane, len, g);
        at_load(t.p, i0, flags & AT_P16, vec, lane, len, p);
        if constexpr (BITS == 32) {
            at_load(t.m, i0, false, vec, lane, len, m);
            at_load(t.v, i0, false, vec, lane, len, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) p[j] = adamw_math(p[j], m[j], v[j], __fmul_rn(g[j], s.grad_scale), flags & AT_DECAY, s.hp, bc1, bc2);
            at_store(t.m, i0, false, vec, lane, len, m);
            at_store(t.v, i0, false, vec, lane, len, v);
        } else {
            const uint2 mc = at_load_codes(t.m, i0, vec, lane, len), vc = at_load_codes(t.v, i0, vec, lane, len);
            const float ms = t.m_scale[tb], vs = t.v_scale[tb];
            at_decode(mc, m);
            at_decode(vc, v);
            uint32_t mtop = 0, vtop = 0;
            const float wd = (flags & AT_DECAY) ? lrwd : 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float gj = __fmul_rn(g[j], s.grad_scale), root = __fmul_rn(v[j], vs);
                m[j] = __fadd_rn(__fmul_rn(s.hp.beta1, __fmul_rn(m[j], ms)), __fmul_rn(omb1, gj));
                v[j] = __fsqrt_rn(__fadd_rn(__fmul_rn(s.hp.beta2, __fmul_rn(root, root)), __fmul_rn(__fmul_rn(omb2, gj), gj)));
                mtop = max(mtop, __float_as_uint(m[j]) & 0x7fffffffu);
                vtop = max(vtop, __float_as_uint(v[j]) & 0x7fffffffu);
                // the root is at hand and the corrections are factors of the step: one approximate division (2 ulp) is left
                const float up = __fdividef(s.hp.lr * (m[j] * rbc1), fmaf(v[j], rroot2, s.hp.eps));
                p[j] = (p[j] - wd * p[j]) - up;
            }
            // elements past the end of a tensor: all their inputs are 0, so they do not touch the maxima
            mtop = __reduce_max_sync(0xffffffffu, mtop);
            vtop = __reduce_max_sync(0xffffffffu, vtop);
            float mscale, vscale, mf, vf;
            at_constant(mtop, mscale, mf);
            at_constant(vtop, vscale, vf);
            const uint32_t key = at_mix(at_mix(step_key + 0x9E3779B9u * (uint32_t)(s.first_tensor + lo + 1)) + (uint32_t)(i0 >> 32));
            uint32_t mo[2] = {0u, 0u}, vo[2] = {0u, 0u};
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t h = at_mix(((uint32_t)i0 + at_elem(vec, lane, j)) ^ key);
                const float rm = fminf(__fmul_rn(fabsf(m[j]), mf), 448.f), rv = fminf(__fmul_rn(v[j], vf), 448.f);
                uint32_t cm = at_code(rm, h & 0xffffu), cv = at_code(rv, h >> 16);
                if (rv > 0.f && cv == 0u) cv = 1u;
                if (m[j] < 0.f) cm |= 0x80u;
                mo[j >> 2] |= cm << (8 * (j & 3));
                vo[j >> 2] |= cv << (8 * (j & 3));
            }
            if (mtop >= 0x7f800000u) { mo[0] = 0u; mo[1] = 0u; }
            if (vtop >= 0x7f800000u) { vo[0] = 0u; vo[1] = 0u; }
            at_store_codes(t.m, i0, vec, lane, len, make_uint2(mo[0], mo[1]));
            at_store_codes(t.v, i0, vec, lane, len, make_uint2(vo[0], vo[1]));
            if (lane == 0) { t.m_scale[tb] = mscale; t.v_scale[tb] = vscale; }
        }
        at_store(t.p, i0, flags & AT_P16, vec, lane, len, p);
    }
}

}  // namespace pac
