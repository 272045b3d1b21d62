// One AdamW step over a list of tensors in one launch, moments in fp32 or in 8 bits.
//
//   m = b1 m + (1-b1) g;  v = b2 v + ((1-b2) g) g;  p = (p - lr wd p) - lr (m / bc1) / (sqrt(v / bc2) + eps)
//
// 8 bits: m and sqrt(v) are kept as float8 (E4M3) times an fp32 constant per 256 elements, absmax / 448.  The root halves
// the range of exponents that has to fit.  With beta2 = 0.999 a step moves v by a thousandth and neighbouring codes are
// an eighth apart, so rounding to the nearest would hold v where it is for ever; codes are rounded up or down by 16
// random bits instead (up with the probability of the remainder), which keeps m and the root unbiased.  v, the root's square, has
// the rounding's variance on top of it: after 4000 steps 5 % too much on average, and 17 % of noise in the root.  The bits are a hash
// of (seed, step, tensor, element): the same call gives the same codes.  A root that is not 0 never becomes 0, so a
// moment never meets a denominator of eps alone; what lies below 1 / 229376 of its block's largest is held too large for that.  A
// block with a gradient that is not finite gets the constant NaN.
//
// The step reads and writes every element once: 28 bytes (fp32 everywhere), 16 (moments in 8 bits), 10 (bf16 parameters
// and gradients on top).  A warp takes 256 elements, eight per lane, so the block's maximum is five shuffles and the
// moments never leave its registers between decoding and encoding.  The list is an argument of the kernel (constant
// memory): nothing to copy, nothing to keep alive after the call, capturable.
//
// Measured, 202 M elements: 512 us with fp32 parameters and 8-bit moments (6.3 TB/s), 459 us with bf16 ones (4.4 TB/s: the
// same 60 instructions an element for half the bytes, 80 % of the issue slots; two blocks ahead do not fit the registers, 487 us and
// more); fp32 everywhere 50 M in 228 us (6.2 TB/s), with bf16 parameters and gradients 197.
#pragma once
#include "pac_ptx.cuh"
#include "pac_adamw.cuh"

namespace pac {

constexpr int AT_BLOCK = 256, AT_SMALL = 48, AT_LARGE = 480, AT_CTAS = 3;
struct AtTensor {
    void* p; const void* g; void* m; void* v;
    float* m_scale; float* v_scale;
    long long n;
    uint32_t first_chunk;       // chunks (AtStep::chunk blocks of 256 elements each) ahead of this tensor's
    uint32_t flags;             // see AT_*
};
constexpr uint32_t AT_P16 = 1u, AT_G16 = 2u, AT_DECAY = 4u, AT_VEC = 8u;
template <int CAP>
struct AtList { AtTensor t[CAP]; };
struct AtStep {
    int count, first_tensor;    // tensors of this launch; the first one's place in the caller's list (names its random bits)
    uint32_t chunks, chunk;     // chunks in all; blocks to a chunk
    pac_adamw hp;
    float bc1, bc2, grad_scale;
    uint32_t seed, step;
    const long long* dev_step;  // when given: the number of the step, in place of step, bc1, bc2
};

// A bijection of 32 bits whose every output bit depends on every input bit: the finaliser of MurmurHash3 (Austin Appleby, public
// domain), two multiplications between xor-shifts, with its published constants.
__host__ __device__ __forceinline__ uint32_t at_mix(uint32_t x) {
    x ^= x >> 16; x *= 0x85EBCA6Bu;
    x ^= x >> 13; x *= 0xC2B2AE35u;
    return x ^ (x >> 16);
}

// Consecutive words in one access; eight values from fp32 or bf16 words.
__device__ __forceinline__ void at_load_words(uint32_t (&x)[8], const char* p) {
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]), "=r"(x[4]), "=r"(x[5]), "=r"(x[6]), "=r"(x[7]) : "l"(p));
}
__device__ __forceinline__ void at_load_words(uint32_t (&x)[4], const char* p) {
    asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "l"(p));
}
__device__ __forceinline__ void at_load_words(uint32_t (&x)[2], const char* p) {
    asm volatile("ld.global.v2.b32 {%0, %1}, [%2];" : "=r"(x[0]), "=r"(x[1]) : "l"(p));
}
__device__ __forceinline__ void at_values(const uint32_t (&w)[8], float (&x)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(w[j]);
}
__device__ __forceinline__ void at_values(const uint32_t (&w)[4], float (&x)[8]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) { x[2 * j] = __uint_as_float(w[j] << 16); x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u); }
}
template <bool IS16>
__device__ __forceinline__ void at_store8(void* base, long long i, const float (&x)[8]) {
    if constexpr (IS16) {
        *reinterpret_cast<uint4*>(static_cast<bf16*>(base) + i) =
            make_uint4(bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7]));
    } else {
        st_global_32(static_cast<float*>(base) + i,
                     make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])),
                     make_uint4(__float_as_uint(x[4]), __float_as_uint(x[5]), __float_as_uint(x[6]), __float_as_uint(x[7])));
    }
}
__device__ __forceinline__ float at_load1(const void* base, long long i, bool is16) {
    return is16 ? __bfloat162float(static_cast<const bf16*>(base)[i]) : static_cast<const float*>(base)[i];
}
__device__ __forceinline__ void at_store1(void* base, long long i, bool is16, float x) {
    if (is16) static_cast<bf16*>(base)[i] = __float2bfloat16(x);
    else static_cast<float*>(base)[i] = x;
}
// Eight E4M3 codes -> fp32 (exact).
__device__ __forceinline__ void at_decode(uint2 c, float (&x)[8]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t w = (j < 2 ? c.x : c.y) >> (16 * (j & 1));
        uint32_t h;
        asm("{\n .reg .b16 t;\n cvt.u16.u32 t, %1;\n cvt.rn.f16x2.e4m3x2 %0, t;\n}" : "=r"(h) : "r"(w));
        asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %2;\n cvt.f32.f16 %0, a;\n cvt.f32.f16 %1, b;\n}" : "=f"(x[2 * j]), "=f"(x[2 * j + 1]) : "r"(h));
    }
}
__device__ __forceinline__ float at_decode1(unsigned char c) {
    float x[8];
    at_decode(make_uint2(c, 0u), x);
    return x[0];
}
// Two fp32 operations in one instruction, each rounded as the scalar one.
struct F2 {
    unsigned long long w;
    __device__ __forceinline__ F2(float x, float y) { asm("mov.b64 %0, {%1, %2};" : "=l"(w) : "f"(x), "f"(y)); }
    __device__ __forceinline__ explicit F2(float x) : F2(x, x) {}
    __device__ __forceinline__ explicit F2(unsigned long long u) : w(u) {}
    __device__ __forceinline__ void get(float& x, float& y) const { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(w)); }
};
__device__ __forceinline__ F2 mul2(F2 a, F2 b) { unsigned long long d; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a.w), "l"(b.w)); return F2(d); }
__device__ __forceinline__ F2 mul2_rz(F2 a, F2 b) { unsigned long long d; asm("mul.rz.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a.w), "l"(b.w)); return F2(d); }
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) { unsigned long long d; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a.w), "l"(b.w), "l"(c.w)); return F2(d); }

// Larger magnitude; a NaN wins.
__device__ __forceinline__ float at_top(float top, float x) {
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(top), "f"(fabsf(x)));
    return d;
}
// Constant of a block and the factor into E4M3's range, from its largest magnitude.
__device__ __forceinline__ void at_constant(float top, float& scale, float& f) {
    if (!(top < __uint_as_float(0x7f800000u))) { scale = __uint_as_float(0x7fffffffu); f = 0.f; }
    else if (top < 7.888609052210118e-31f) { scale = 0.f; f = 0.f; }            // 2^-100: 448 / top would overflow further down
    else { scale = __fdiv_rn(top, 448.f); f = __fdiv_rn(448.f, top); }
}
// E4M3 codes (without signs) of two numbers x f of magnitude up to 448, in the top bytes, rounded up with the probability of
// what is cut off; a0, a1: 16 random bits each in the middle two bytes.  E4M3's exponents are those of fp32 moved by 120 and its
// subnormals are then fp32's, so after a (truncating) factor of 2^-120 the code is what stands above bit 20 of the number, small
// or not; the shift drops the sign.  (x f may exceed 448 by an ulp or two: less than what the random bits leave below a carry.)
__device__ __forceinline__ void at_codes2(F2 x, F2 f, uint32_t a0, uint32_t a1, uint32_t& c0, uint32_t& c1) {
    float r0, r1;
    mul2_rz(mul2(x, f), F2(7.52316384526264e-37f)).get(r0, r1);
    c0 = (__float_as_uint(r0) << 4) + a0;
    c1 = (__float_as_uint(r1) << 4) + a1;
}
// Top bytes of four words.
__device__ __forceinline__ uint32_t at_pack(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0073), __byte_perm(c, d, 0x0073), 0x5410);
}

// What every element of a launch shares.
struct AtConst {
    float lrbc1, rroot2, omb1, omb2, lrwd, bc1, bc2;
    uint32_t step_key;
};

// The 8-bit update of two elements: m and the root come decoded but for their block's constant, and leave as fp32.  The root is
// that of v for 0 and from 2^-126 to the largest number; at_update1 is for the rest.
__device__ __forceinline__ void at_update2(float* p, float* m, float* v, const float* g, float ms, float vs, float wd, const AtStep& s, const AtConst& c) {
    const F2 gg = mul2(F2(g[0], g[1]), F2(s.grad_scale)), root = mul2(F2(v[0], v[1]), F2(vs));
    // every rounding as written above (the sums are scalar: the compiler fuses a packed sum with the product before it)
    float a[2], b[2], d[2], e[2];
    mul2(F2(s.hp.beta1), mul2(F2(m[0], m[1]), F2(ms))).get(a[0], a[1]);
    mul2(F2(c.omb1), gg).get(b[0], b[1]);
    mul2(F2(s.hp.beta2), mul2(root, root)).get(d[0], d[1]);
    mul2(mul2(F2(c.omb2), gg), gg).get(e[0], e[1]);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        m[k] = __fadd_rn(a[k], b[k]);
        v[k] = __fadd_rn(d[k], e[k]);
        asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(d[k]) : "f"(fmaxf(v[k], 1.17549435e-38f)));
    }
    // sqrt(v): the hardware's y = 1 / sqrt(v) and one step of Newton's method on r^2 = v in fused arithmetic, r = vy,
    // r + (v - r^2) y / 2, which leaves 2^-45 before its rounding.  (With the hardware's approximate root and fused sums 7 %
    // less time, but codes and constants that differ from the definition's here and there.)
    const F2 y(d[0], d[1]), vv(v[0], v[1]), r = mul2(vv, y), nr = mul2(vv, mul2(y, F2(-1.f)));
    fma2(fma2(nr, r, vv), mul2(y, F2(0.5f)), r).get(v[0], v[1]);
    // the root is at hand for the step too, whose corrections are factors: a reciprocal (1 ulp) is left
    fma2(F2(v[0], v[1]), F2(c.rroot2), F2(s.hp.eps)).get(d[0], d[1]);
#pragma unroll
    for (int k = 0; k < 2; ++k) asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(d[k]) : "f"(d[k]));
    const F2 pp(p[0], p[1]);
    fma2(mul2(F2(-c.lrbc1), F2(m[0], m[1])), F2(d[0], d[1]), fma2(F2(-wd), pp, pp)).get(p[0], p[1]);
}
// The same of element i from what is in memory, with a root that is right over all of fp32's range (subnormal v; v = infinity, whose
// step is none).
__device__ __forceinline__ float3 at_update1(const AtTensor& t, long long i, float ms, float vs, float wd, const AtStep& s, const AtConst& c) {
    const float g = __fmul_rn(at_load1(t.g, i, t.flags & AT_G16), s.grad_scale), p = at_load1(t.p, i, t.flags & AT_P16);
    const float m0 = __fmul_rn(at_decode1(static_cast<const unsigned char*>(t.m)[i]), ms), root = __fmul_rn(at_decode1(static_cast<const unsigned char*>(t.v)[i]), vs);
    const float m = __fadd_rn(__fmul_rn(s.hp.beta1, m0), __fmul_rn(c.omb1, g));
    const float v = __fsqrt_rn(__fadd_rn(__fmul_rn(s.hp.beta2, __fmul_rn(root, root)), __fmul_rn(__fmul_rn(c.omb2, g), g)));
    return make_float3(__fmaf_rn(__fmul_rn(-c.lrbc1, m), __fdiv_rn(1.f, __fmaf_rn(v, c.rroot2, s.hp.eps)), __fmaf_rn(-wd, p, p)), m, v);
}
// Whether elements need it, from the largest of their roots.  A v below 2^-126 beside a root of 2^-40 or more does not: its
// code is the smallest whatever its root (below 2^-18 of the block's largest it is rounded to 0 or that, and 0 becomes that), and in
// the step eps hides a root below 2^-63 / sqrt(bc2), but for an eps below 2^25 times that (TINY: 1.2e-10 for beta2 = 0.999): then
// every root is looked at.  (In every kernel that took the listed sizes 1 to 2 us more: 8.7 M elements 25 and 27 us.)  Blocks of
// zeros do not come here, and in training hardly any do.
__device__ __forceinline__ bool at_extreme(float top) { return !(top < __uint_as_float(0x7f800000u)) || (top < 9.094947e-13f && top > 0.f); }
__device__ __forceinline__ bool at_small(float root) { return root < 1.08420217e-19f && root > 0.f; }    // 2^-63

// Random bits of one element: the hash of its number ^ the block's key, from where the first xor-shift is done (x1).
__device__ __forceinline__ uint32_t at_random(uint32_t x1) {
    uint32_t h = x1 * 0x85EBCA6Bu;
    h = (h ^ (h >> 13)) * 0xC2B2AE35u;
    return h ^ (h >> 16);
}
// Codes of two elements in the top bytes of words.
__device__ __forceinline__ void at_encode2(const float* m, const float* v, float mf, float vf, uint32_t x1, uint32_t y1, uint32_t* mo, uint32_t* vo) {
    const uint32_t h0 = at_random(x1), h1 = at_random(y1);
    at_codes2(F2(m[0], m[1]), F2(mf), __byte_perm(h0, 0u, 0x4104), __byte_perm(h1, 0u, 0x4104), mo[0], mo[1]);
    at_codes2(F2(v[0], v[1]), F2(vf), __byte_perm(h0, 0u, 0x4324), __byte_perm(h1, 0u, 0x4324), vo[0], vo[1]);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        // a moment of -0 has no sign; a root above 0 is at least 2^-75, its bits are above 2^24, and its code is not 0
        mo[e] |= m[e] < 0.f ? 0x80000000u : 0u;
        vo[e] = max(vo[e], min(__float_as_uint(v[e]), 0x01000000u));
    }
}
__device__ __forceinline__ bool at_finite(float top) { return top < __uint_as_float(0x7f800000u); }
__device__ __forceinline__ float at_warp_top(float top) { return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top))); }

// The update of one element (and of a second one of zeros) from what is in memory.
__device__ __forceinline__ void at_again(const AtTensor& t, long long i, bool g16, float ms, float vs, float wd, const AtStep& s, const AtConst& c,
                                         float (&p)[2], float (&m)[2], float (&v)[2]) {
    const float g[2] = {at_load1(t.g, i, g16), 0.f};
    m[0] = at_decode1(static_cast<const unsigned char*>(t.m)[i]);
    v[0] = at_decode1(static_cast<const unsigned char*>(t.v)[i]);
    m[1] = v[1] = 0.f;
    at_update2(p, m, v, g, ms, vs, wd, s, c);
    if (at_extreme(v[0]) || at_small(v[0])) {
        const float3 u = at_update1(t, i, ms, vs, wd, s, c);
        p[0] = u.x; m[0] = u.y; v[0] = u.z;
    }
}
// Up to 256 elements at any alignment, one of each 32 per lane.  8 bits: the moments are formed twice, for the maximum and for
// the codes, from what is still in memory.
template <int BITS>
__device__ __forceinline__ void at_block_any(const AtTensor& t, long long tb, uint32_t tensor_key, const AtStep& s, const AtConst& c) {
    const int lane = threadIdx.x & 31;
    const long long i0 = tb * AT_BLOCK;
    const int len = (int)min((long long)AT_BLOCK, t.n - i0);
    const bool p16 = t.flags & AT_P16, g16 = t.flags & AT_G16;
    if constexpr (BITS == 32) {
        float *mp = static_cast<float*>(t.m), *vp = static_cast<float*>(t.v);
#pragma unroll 2
        for (int e = lane; e < len; e += 32) {
            float m = mp[i0 + e], v = vp[i0 + e];
            const float p = adamw_math(at_load1(t.p, i0 + e, p16), m, v, __fmul_rn(at_load1(t.g, i0 + e, g16), s.grad_scale), t.flags & AT_DECAY, s.hp, c.bc1, c.bc2);
            mp[i0 + e] = m;
            vp[i0 + e] = v;
            at_store1(t.p, i0 + e, p16, p);
        }
    } else {
        unsigned char *mp = static_cast<unsigned char*>(t.m), *vp = static_cast<unsigned char*>(t.v);
        const float ms = t.m_scale[tb], vs = t.v_scale[tb], wd = (t.flags & AT_DECAY) ? c.lrwd : 0.f;
        float mtop = 0.f, vtop = 0.f, mscale, vscale, mf, vf;
#pragma unroll 2
        for (int e = lane; e < len; e += 32) {
            float m[2], v[2], p[2] = {at_load1(t.p, i0 + e, p16), 0.f};
            at_again(t, i0 + e, g16, ms, vs, wd, s, c, p, m, v);
            at_store1(t.p, i0 + e, p16, p[0]);
            mtop = at_top(mtop, m[0]);
            vtop = at_top(vtop, v[0]);
        }
        mtop = at_warp_top(mtop);
        vtop = at_warp_top(vtop);
        at_constant(mtop, mscale, mf);
        at_constant(vtop, vscale, vf);
        const uint32_t key = at_mix(tensor_key + (uint32_t)(i0 >> 32));
#pragma unroll 2
        for (int e = lane; e < len; e += 32) {
            float m[2], v[2], p[2] = {0.f, 0.f};
            at_again(t, i0 + e, g16, ms, vs, wd, s, c, p, m, v);
            const uint32_t x0 = ((uint32_t)i0 + e) ^ key;
            uint32_t mo[2], vo[2];
            at_encode2(m, v, mf, vf, x0 ^ (x0 >> 16), 0u, mo, vo);
            mp[i0 + e] = at_finite(mtop) ? (unsigned char)(mo[0] >> 24) : 0;
            vp[i0 + e] = at_finite(vtop) ? (unsigned char)(vo[0] >> 24) : 0;
        }
        __syncwarp();                                        // every lane has read the old constants
        if (lane == 0) { t.m_scale[tb] = mscale; t.v_scale[tb] = vscale; }
    }
}

// 256 elements by a warp, eight consecutive ones per lane; all pointers aligned to eight elements.  What is read of a block,
// as it lies in memory: the next block's are on their way while this one is computed (8 bits, 202 M bf16 elements: 697 us
// without).
template <int BITS, bool P16, bool G16>
struct AtRaw {
    uint32_t p[P16 ? 4 : 8], g[G16 ? 4 : 8], m[BITS == 32 ? 8 : 2], v[BITS == 32 ? 8 : 2];
    float ms, vs;
    __device__ __forceinline__ void load(const AtTensor& t, long long tb) {
        const long long i = tb * AT_BLOCK + (threadIdx.x & 31) * 8;
        at_load_words(g, static_cast<const char*>(t.g) + i * (G16 ? 2 : 4));
        at_load_words(p, static_cast<const char*>(t.p) + i * (P16 ? 2 : 4));
        at_load_words(m, static_cast<const char*>(t.m) + i * (BITS == 32 ? 4 : 1));
        at_load_words(v, static_cast<const char*>(t.v) + i * (BITS == 32 ? 4 : 1));
        if constexpr (BITS == 8) { ms = t.m_scale[tb]; vs = t.v_scale[tb]; }
    }
};
template <int BITS, bool P16, bool G16, bool TINY>
__device__ __forceinline__ bool at_block(const AtTensor& t, long long tb, const AtRaw<BITS, P16, G16>& raw, uint32_t tensor_key, const AtStep& s, const AtConst& c) {
    const int lane = threadIdx.x & 31;
    const long long i = tb * AT_BLOCK + lane * 8;
    float p[8], g[8], m[8], v[8];
    at_values(raw.g, g);
    at_values(raw.p, p);
    if constexpr (BITS == 32) {
        at_values(raw.m, m);
        at_values(raw.v, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) p[j] = adamw_math(p[j], m[j], v[j], __fmul_rn(g[j], s.grad_scale), t.flags & AT_DECAY, s.hp, c.bc1, c.bc2);
        at_store8<false>(t.m, i, m);
        at_store8<false>(t.v, i, v);
        at_store8<P16>(t.p, i, p);
    } else {
        const float wd = (t.flags & AT_DECAY) ? c.lrwd : 0.f;
        at_decode(make_uint2(raw.m[0], raw.m[1]), m);
        at_decode(make_uint2(raw.v[0], raw.v[1]), v);
        float mtop = 0.f, vtop = 0.f, mscale, vscale, mf, vf;
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            at_update2(p + j, m + j, v + j, g + j, raw.ms, raw.vs, wd, s, c);
            mtop = at_top(at_top(mtop, m[j]), m[j + 1]);
            vtop = at_top(at_top(vtop, v[j]), v[j + 1]);
        }
        bool again = false;
        if constexpr (TINY) {
#pragma unroll
            for (int j = 0; j < 8; ++j) again |= at_small(v[j]);
        }
        mtop = at_warp_top(mtop);
        vtop = at_warp_top(vtop);
        if (at_extreme(vtop) || (TINY && __any_sync(0xffffffffu, again))) {
            return false;
        }
        at_store8<P16>(t.p, i, p);
        at_constant(mtop, mscale, mf);
        at_constant(vtop, vscale, vf);
        // the hash of element ^ key; a lane's elements differ in the low byte only, so its first xor-shift is done once
        const uint32_t x0 = (uint32_t)i ^ at_mix(tensor_key + (uint32_t)(i >> 32)), x1 = x0 ^ (x0 >> 16);
        uint32_t mo[8], vo[8];
#pragma unroll
        for (int j = 0; j < 8; j += 2) at_encode2(m + j, v + j, mf, vf, x1 ^ (uint32_t)j, x1 ^ (uint32_t)(j + 1), mo + j, vo + j);
        *reinterpret_cast<uint2*>(static_cast<unsigned char*>(t.m) + i) =
            at_finite(mtop) ? make_uint2(at_pack(mo[0], mo[1], mo[2], mo[3]), at_pack(mo[4], mo[5], mo[6], mo[7])) : make_uint2(0u, 0u);
        *reinterpret_cast<uint2*>(static_cast<unsigned char*>(t.v) + i) =
            at_finite(vtop) ? make_uint2(at_pack(vo[0], vo[1], vo[2], vo[3]), at_pack(vo[4], vo[5], vo[6], vo[7])) : make_uint2(0u, 0u);
        if (lane == 0) { t.m_scale[tb] = mscale; t.v_scale[tb] = vscale; }
    }
    return true;
}
template <int BITS, bool P16, bool G16, bool TINY>
__device__ __forceinline__ uint32_t at_blocks(const AtTensor& t, const long long first, long long end, uint32_t tensor_key, const AtStep& s, const AtConst& c) {
    uint32_t left = 0;
    long long tb = first;
    AtRaw<BITS, P16, G16> now;
    if constexpr (BITS == 32) {                             // little to compute, and twice the words would not fit the registers
#pragma unroll 1
        for (; tb < end; ++tb) {
            now.load(t, tb);
            at_block<BITS, P16, G16, TINY>(t, tb, now, tensor_key, s, c);
        }
    } else {
        now.load(t, tb);
        AtRaw<BITS, P16, G16> next = now;
#pragma unroll 1
        for (; tb < end; ++tb) {
            if (tb + 1 < end) next.load(t, tb + 1);
            if (!at_block<BITS, P16, G16, TINY>(t, tb, now, tensor_key, s, c)) left |= 1u << (tb - first);
            now = next;
        }
    }
    return left;
}
template <int BITS, int CAP, bool TINY>
__global__ void __launch_bounds__(256, AT_CTAS) adamw_tensors_kernel(const __grid_constant__ AtList<CAP> list, const __grid_constant__ AtStep s) {
    __shared__ float bc_sh[2];
    AtConst k;
    uint32_t step = s.step;
    k.bc1 = s.bc1; k.bc2 = s.bc2;
    if (s.dev_step) {
        const long long st = *s.dev_step;
        step = (uint32_t)st;
        if (threadIdx.x < 2) bc_sh[threadIdx.x] = (float)(1.0 - pow((double)(threadIdx.x ? s.hp.beta2 : s.hp.beta1), (double)st));
        __syncthreads();
        k.bc1 = bc_sh[0]; k.bc2 = bc_sh[1];
    }
    k.lrbc1 = __fdiv_rn(s.hp.lr, k.bc1);
    k.rroot2 = __fdiv_rn(1.f, __fsqrt_rn(k.bc2));
    k.omb1 = __fsub_rn(1.f, s.hp.beta1);
    k.omb2 = __fsub_rn(1.f, s.hp.beta2);
    k.lrwd = __fmul_rn(s.hp.lr, s.hp.weight_decay);
    k.step_key = BITS == 8 ? at_mix(s.seed + 0x9E3779B9u * step) : 0u;
    const uint32_t warps = (gridDim.x * blockDim.x) >> 5;
    for (uint32_t c = (blockIdx.x * blockDim.x + threadIdx.x) >> 5; c < s.chunks; c += warps) {
        int lo = 0, hi = s.count - 1;                       // the last tensor that begins at or before chunk c
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (list.t[mid].first_chunk <= c) lo = mid; else hi = mid - 1;
        }
        const AtTensor& t = list.t[lo];
        const uint32_t tensor_key = BITS == 8 ? at_mix(k.step_key + 0x9E3779B9u * (uint32_t)(s.first_tensor + lo + 1)) : 0u;
        const long long first = (long long)(c - t.first_chunk) * s.chunk, last = t.n / AT_BLOCK;
        const long long end = min(first + s.chunk, (t.n + AT_BLOCK - 1) / AT_BLOCK);
        const long long whole = (t.flags & AT_VEC) ? min(end, last) : first;
        uint32_t left = 0;                                  // blocks ahead of `whole` that have yet to be done
        if (first < whole) {
            if (t.flags & AT_P16) {
                if (t.flags & AT_G16) left = at_blocks<BITS, true, true, TINY>(t, first, whole, tensor_key, s, k);
                else left = at_blocks<BITS, true, false, TINY>(t, first, whole, tensor_key, s, k);
            } else {
                if (t.flags & AT_G16) left = at_blocks<BITS, false, true, TINY>(t, first, whole, tensor_key, s, k);
                else left = at_blocks<BITS, false, false, TINY>(t, first, whole, tensor_key, s, k);
            }
        }
#pragma unroll 1
        for (long long tb = left ? first : whole; tb < end; ++tb)
            if (tb >= whole || (left >> (tb - first) & 1u)) at_block_any<BITS>(t, tb, tensor_key, s, k);
    }
}

}  // namespace pac
