// Products with a frozen matrix W [N][K] in MXFP4 (pac_mxfp.cuh), the other operand as it is:
//     y  = x W^T      [M][N]      (GRAD = false; reduction over the columns of W)
//     dx = dy W       [M][K]      (GRAD = true;  reduction over the rows of W; W is frozen, so this is the whole backward pass)
//
// A value of W is a bf16 exactly (two significant bits times a power of two), so W goes through the bf16 tensor cores
// without an error of its own: converter warps turn codes into a bf16 tile in shared memory, tcgen05.mma takes it from
// there.  W is the M operand (128 of its rows, or of its columns, per CTA) and the tokens are the N operand: few tokens
// cost few columns, each code is converted once per CTA however many tokens there are, and in the accumulator a lane is
// an output column, so that a warp's store is 32 neighbours of a row of y without a detour through shared memory.
//
// Both directions walk W in pieces of 128 rows x 128 columns: 8 KB of codes and 512 bytes of scales, two K steps of 64.
// Forward the tile is K-major (a thread converts one block of 32 of a row), backward MN-major (the same block lies along
// the M dimension): the same 64 bytes go to another place, and the descriptor says so.
//
// Few tiles: the reduction is split over a cluster, whose CTAs then add their partial sums through distributed shared
// memory in the order of their ranks (no atomics, no workspace).
//
// What bounds it: converting, as long as there are few tokens to a tile.  A value costs two byte permutations, three masks or
// shifts (a half-rate pipe) and half a product, so 32000 x 4096 takes 25 us of that pipe alone and 52 us in two uneven waves
// of 250 CTAs (17 to 32 tokens; backward in one wave of split reductions 49); 4096 x 4096 takes 12 us.  From some 100 tokens on the
// tensor cores: see pac_mxfp_pair.cuh.
//
// Precision: operands exact, sums in fp32.  The tensor core cuts partial sums instead of rounding them, so K steps take
// turns over the accumulators that tensor memory has room for (MX_ADDS_F32 below).  x in fp32 enters as three bf16 terms that
// add up to it exactly (below 2^-110 the third one ends at bf16's smallest number: to 2^-134); the second and third share an
// accumulator, whose additions are twice as many and cut 2^-8 as much.
#pragma once
#include <cooperative_groups.h>

#include "pac_mxfp.cuh"

namespace pac {

constexpr int ML_BK = 64;                                   // reduction elements per stage
constexpr int ML_CONV_WARPS = 16;                            // in groups of four, each with every fourth step
constexpr uint32_t ML_A_BYTES = 128 * ML_BK * 2;
constexpr uint32_t ML_CODE_BYTES = 128 * 64 + MX_SCALE_PIECE;
constexpr int ML_MAX_STAGES = 8, ML_MAX_CODES = 8;
// Pieces of codes in flight.  A group of converting warps has every second piece, so with an even number it meets a place of the
// ring at every one of its fills, and the parity that it waits for is that of the fill it means; with an odd number it would
// pass over fills, and a wait could be answered by the phase before the one that it passed over.
constexpr int ML_CODES = 6, ML_CODES_WIDE = 2;
static_assert(ML_CODES % (ML_CONV_WARPS / 8) == 0 && ML_CODES_WIDE % (ML_CONV_WARPS / 8) == 0 && ML_MAX_STAGES % (ML_CONV_WARPS / 4) == 0 && 4 % (ML_CONV_WARPS / 4) == 0,
              "every group of converting warps meets its places of the rings at every fill");
constexpr size_t ML_SMEM_MOST = 232448 - 1024 - 512;
// Additions (of 16 products each, 64 in the block-scaled product) that an accumulator takes: each cuts up to 2^-23 of the sum, always
// towards zero, so the cuts add up over the length of a reduction.  128 take at most 2^-16 of the sums from an fp32 result, 512 at
// most 2^-14 from a bf16 one, a 64th of the half step that it is rounded by.  (All 2000 of a gradient over 32000 rows in one:
// 1.4 in 1000 of its bf16 values on the other side of the exact one's rounding, 0.4 in 1000 so, 0.2 in 1000 of an fp32 sum's.)
constexpr int MX_ADDS_F32 = 128, MX_ADDS_BF16 = 512;

// What becomes of a product's accumulators (the block-scaled product's as well).
struct MxOut {
    void* y; long long ldy; int y_f32;
    int M;                                                  // tokens
    int cols;                                               // columns of y
    int nt;                                                 // tokens per tile, a multiple of 16
    int split;                                              // CTAs of a cluster that share a tile's reduction
    int n_acc;                                              // accumulators of nt columns
    int terms;                                              // y is the sum of so many rows M apart (1: as it is)
};
struct MlParams {
    MxOut o;
    const unsigned char* scales;
    int red;                                                // length of the reduction: K, or N with GRAD
    int pieces;                                             // pieces of scales per row tile
    int red_tiles;                                          // ceil(red / 128)
    int stages, code_stages;
    uint32_t stage_bytes, code_at;                          // bytes per stage; offset of the ring of codes
    uint32_t tmem_cols;
    int x_rows;                                             // rows of a term of x
    bool after;                                             // launched ahead of the end of the kernel that packs x
};

__device__ __forceinline__ void ml_tma_2d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1) : "memory");
}
__device__ __forceinline__ void sts128(uint32_t a, uint4 v) { asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory"); }
__device__ __forceinline__ uint4 lds128(uint32_t a) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
    uint32_t v;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}

__device__ __forceinline__ float4 add4(float4 a, float4 b) { return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w); }
template <int RANKS, typename Cluster>
__device__ __forceinline__ float4 sum_ranks(Cluster& cluster, float4* part, int i) {
    float4 u[RANKS];
#pragma unroll
    for (int k = 0; k < RANKS; ++k) u[k] = cluster.map_shared_rank(part, k)[i];
#pragma unroll
    for (int k = 1; k < RANKS; ++k) u[0] = add4(u[0], u[k]);
    return u[0];
}

// A column of up to 16 tokens.  The pointer moves on by the pitch: with an address formed for every token (a 64-bit product and a
// test each) a store took a warp 94 clocks and a tile of 256 tokens 12 us.
template <typename T>
__device__ __forceinline__ void mx_store16(T* y, long long ldy, int n, const float (&v)[16]) {
    char* p = reinterpret_cast<char*>(y);
    const long long pitch = ldy * (long long)sizeof(T);
    auto put = [&](float x) {
        if constexpr (sizeof(T) == 4) *reinterpret_cast<float*>(p) = x;
        else *reinterpret_cast<bf16*>(p) = __float2bfloat16(x);
        p += pitch;
    };
    if (n >= 16) {
#pragma unroll
        for (int e = 0; e < 16; ++e) put(v[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 15; ++e)
            if (e < n) put(v[e]);
    }
}
// Accumulators -> y, by all threads of the CTA.  A lane is an output column and an accumulator column a token, so a warp
// stores 32 neighbours of a row of y; warps 2-9, two per quadrant of lanes, share the tokens.  A tile whose reduction is
// split goes through shared memory and is added up by the cluster, rank by rank.  `used`: accumulators that some step has
// written; `last`: the last one has been written in any case.  last_word(token, column, sum) is what is stored of shared sums.
template <typename Last>
__device__ __forceinline__ void mx_finish(const MxOut& o, uint32_t tmem_base, unsigned char* smem, uint32_t accf, volatile int* abort_flag, int wt, int t0,
                                          int rank, int used, bool last, Last last_word) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int n_tok = min(o.nt, o.M - t0);
    const bool shared = o.split > 1 || o.terms > 1;
    if (warp >= 2 && warp < 10) {
        const bool ok = mbar_wait_uniform(accf, 0, abort_flag, nullptr);
        if (!ok) drain_after_abort(abort_flag);              // copies in flight land before their memory is written again
        tc_fence_after();
        const int q = warp & 3, half = (warp - 2) >> 2;
        const int col = wt * 128 + q * 32 + lane;
        const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16);
        float* part = reinterpret_cast<float*>(smem) + q * 32 + lane;
        const float bad = __uint_as_float(0x7fffffffu);      // a wait that ran out leaves NaN, not a wrong number
        const int most = min(o.n_acc, used);
        for (int c0 = half * 16; c0 < o.nt; c0 += 32) {
            float v[16], w[16];
            tmem_ld16(taddr + c0, v);
            tmem_ld_wait();
            for (int a = 1; a < most; ++a) {
                tmem_ld16(taddr + a * o.nt + c0, w);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 16; ++e) v[e] += w[e];
            }
            if (last && most < o.n_acc) {
                tmem_ld16(taddr + (o.n_acc - 1) * o.nt + c0, w);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 16; ++e) v[e] += w[e];
            }
            if (!ok) {
#pragma unroll
                for (int e = 0; e < 16; ++e) v[e] = bad;
            }
            if (shared) {
#pragma unroll
                for (int e = 0; e < 16; ++e) part[(c0 + e) * 128] = v[e];
            } else if (col < o.cols) {
                if (o.y_f32) mx_store16(static_cast<float*>(o.y) + (long long)(t0 + c0) * o.ldy + col, o.ldy, n_tok - c0, v);
                else mx_store16(static_cast<bf16*>(o.y) + (long long)(t0 + c0) * o.ldy + col, o.ldy, n_tok - c0, v);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (!shared) return;
    // groups of four columns of a token, 32 to a token
    float4* part = reinterpret_cast<float4*>(smem);
    const int groups = n_tok * 32;
    if (o.terms > 1) {
        // the smallest terms first
        for (int i = threadIdx.x; i < groups; i += blockDim.x) {
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 12
            for (int t = o.terms - 1; t >= 0; --t) v = add4(v, part[t * o.M * 32 + i]);
            part[i] = v;
        }
    }
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    if (o.split > 1) cluster.sync();
    else __syncthreads();
    const int g0 = (int)((long long)groups * rank / o.split), g1 = (int)((long long)groups * (rank + 1) / o.split);
    for (int i = g0 + (int)threadIdx.x; i < g1; i += (int)blockDim.x) {
        const int c = i >> 5, col = wt * 128 + (i & 31) * 4;
        if (col >= o.cols) continue;                         // before anything is loaded: see the end
        float4 v;
        switch (o.split) {                                   // all ranks' parts are asked for before the first is added
            case 2: v = sum_ranks<2>(cluster, part, i); break;
            case 4: v = sum_ranks<4>(cluster, part, i); break;
            case 8: v = sum_ranks<8>(cluster, part, i); break;
            default: v = part[i];
        }
        const float w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (col + e >= o.cols) continue;
            const long long at = (long long)(t0 + c) * o.ldy + col + e;
            const float y = last_word(t0 + c, col + e, w[e]);
            if (o.y_f32) static_cast<float*>(o.y)[at] = y;
            else static_cast<bf16*>(o.y)[at] = __float2bfloat16(y);
        }
    }
    // nobody leaves while its partial sums are still read.  Every load of another CTA's memory above feeds a store, which is issued
    // ahead of the arrival and only once the load has come back; so the arrival needs no release, which would wait for the stores
    // of y as well (1500 clocks)
    if (o.split > 1) {
        __syncwarp();
        asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    }
}

// x as TMA boxes can read it: TERMS matrices [rows][16-byte rows of whole 128-column pieces] in bf16, below one another.  A bf16 x
// whose rows do not begin on 16-byte boundaries is copied; an fp32 x becomes three bf16 terms that add up to it (see above).
__host__ __device__ inline int pack_columns(int red) { return (red + 127) / 128 * 128; }
template <typename T>
__global__ void __launch_bounds__(256) pack_tokens_kernel(const T* __restrict__ x, int M, int red, long long ldx, bool vec, bf16* __restrict__ out) {
    pdl_trigger();
    const int cols = pack_columns(red), groups = cols / 8;
    const long long items = (long long)M * groups, term = (long long)M * cols;
    for (long long it = (long long)blockIdx.x * blockDim.x + threadIdx.x; it < items; it += (long long)gridDim.x * blockDim.x) {
        const long long m = it / groups;
        const int c0 = (int)(it - m * groups) * 8;
        const T* p = x + m * ldx + c0;
        float v[8];
        if (sizeof(T) == 4 && vec && c0 + 8 <= red) {
            const float4 a = *reinterpret_cast<const float4*>(p), b = *(reinterpret_cast<const float4*>(p) + 1);
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = c0 + e < red ? to_f32(p[e]) : 0.f;
        }
        uint32_t h[4], l[4], t[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            h[e] = bf16_pair(v[2 * e], v[2 * e + 1]);
            if constexpr (sizeof(T) == 4) {
                float r[2];
#pragma unroll
                for (int f = 0; f < 2; ++f) {
                    const float x1 = v[2 * e + f];
                    const bool finite = fabsf(x1) < __uint_as_float(0x7f800000u);
                    // the largest values round to an infinity: one step less; an infinity or a NaN is its own first term
                    if (finite && ((h[e] >> (16 * f)) & 0x7fffu) == 0x7f80u) h[e] -= 1u << (16 * f);
                    r[f] = finite ? x1 - __uint_as_float(f ? h[e] & 0xffff0000u : h[e] << 16) : 0.f;
                }
                l[e] = bf16_pair(r[0], r[1]);
                t[e] = bf16_pair(r[0] - __uint_as_float(l[e] << 16), r[1] - __uint_as_float(l[e] & 0xffff0000u));
            }
        }
        bf16* dst = out + m * cols + c0;
        *reinterpret_cast<uint4*>(dst) = make_uint4(h[0], h[1], h[2], h[3]);
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<uint4*>(dst + term) = make_uint4(l[0], l[1], l[2], l[3]);
            *reinterpret_cast<uint4*>(dst + 2 * term) = make_uint4(t[0], t[1], t[2], t[3]);
        }
    }
}

// Codes -> a K step's bf16 tile.  Four warps take a step, the groups of four in turn, so that a warp has several steps' time
// for the waits and fences of one; a thread takes two blocks of 32.  Forward: the step's 64 columns of row `t`; backward: half of
// the 128 columns of row h * 64 + t / 2 (the other 64 are another thread's).  The copy of the codes swizzles their 16-byte
// blocks over 512 bytes, and odd threads begin with their second block backward, so that neither the reads nor the writes
// of eight neighbours meet in a bank.
template <bool GRAD>
struct MlBlocks {
    uint4 c[2];
    uint32_t f[2];
    __device__ __forceinline__ static int row(int t, int h) { return GRAD ? h * 64 + (t >> 1) : t; }
    __device__ __forceinline__ static int block(int t, int h, int i) { return GRAD ? (t & 1) * 2 + (i ^ (t & 1)) : h * 2 + i; }
    // src: a piece of codes and its scales; kt: the piece along the reduction of length red
    __device__ __forceinline__ void load(uint32_t src, int t, int h, int kt, int red) {
        const int r = row(t, h);
        const uint32_t scales = lds32(src + 128 * 64 + mx_scale_at((uint32_t)r, 0u));
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int b = block(t, h, i);
            c[i] = lds128(src + r * 64 + (((uint32_t)b ^ (((uint32_t)r >> 1) & 3u)) << 4));
            // beyond the reduction the codes are 0 and the scale is whatever fills the piece: it must not be a NaN
            const bool in = GRAD ? kt * 128 + r < red : kt * 128 + b * 32 < red;
            f[i] = in ? mx_scale_bf16x2((scales >> (8 * b)) & 255u) : 0u;
        }
    }
    __device__ __forceinline__ void convert(uint32_t (&o)[2][4][4]) const {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t w[4] = {c[i].x, c[i].y, c[i].z, c[i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                mx_bf16x8(w[j], o[i][j]);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[i][j][e] = mul_bf16x2(o[i][j][e], f[i]);
            }
        }
    }
    __device__ __forceinline__ static void store(uint32_t tile, int t, int h, const uint32_t (&o)[2][4][4]) {
        const uint32_t r = (uint32_t)(GRAD ? t >> 1 : t), dst = tile + (GRAD ? (uint32_t)(t & 1) * 8192u : 0u) + r * 128u;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t chunk0 = (uint32_t)(block(t, h, i) & 1) * 4u;
#pragma unroll
            for (int j = 0; j < 4; ++j) sts128(dst + (((chunk0 + j) ^ (r & 7u)) << 4), make_uint4(o[i][j][0], o[i][j][1], o[i][j][2], o[i][j][3]));
        }
    }
};

// Warps: 0 copies, 1 MMAs, 2-17 convert W, 2-9 store y.
template <bool GRAD, int TERMS>
__global__ void __launch_bounds__(32 * (2 + ML_CONV_WARPS), 1)
mxfp_linear_kernel(const __grid_constant__ CUtensorMap map_codes, const __grid_constant__ CUtensorMap map_x, const __grid_constant__ MlParams p) {
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = (unsigned char*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    __shared__ __align__(8) unsigned long long bars[3 * ML_MAX_STAGES + 2 * ML_MAX_CODES + 1];
    __shared__ uint32_t tmem_base_sh;
    __shared__ int abort_sh;
    const uint32_t xfull0 = smem_u32(&bars[0]), afull0 = smem_u32(&bars[ML_MAX_STAGES]), empty0 = smem_u32(&bars[2 * ML_MAX_STAGES]);
    const uint32_t cfull0 = smem_u32(&bars[3 * ML_MAX_STAGES]), cempty0 = smem_u32(&bars[3 * ML_MAX_STAGES + ML_MAX_CODES]);
    const uint32_t accf = smem_u32(&bars[3 * ML_MAX_STAGES + 2 * ML_MAX_CODES]);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = p.o.split > 1 ? (int)(blockIdx.x % p.o.split) : 0;
    const int wt = blockIdx.x / p.o.split, t0 = blockIdx.y * p.o.nt;
    const int kt0 = (int)((long long)p.red_tiles * rank / p.o.split), kt1 = (int)((long long)p.red_tiles * (rank + 1) / p.o.split);
    const int steps = 2 * (kt1 - kt0);
    const uint32_t ring0 = smem_u32(smem), codes0 = ring0 + p.code_at;
    const uint32_t term_bytes = (uint32_t)p.o.nt * 128u;

    if (threadIdx.x == 0) {
        abort_sh = 0;
        for (int s = 0; s < p.stages; ++s) { mbar_init(xfull0 + 8 * s, 1); mbar_init(afull0 + 8 * s, 4); mbar_init(empty0 + 8 * s, 1); }
        for (int s = 0; s < p.code_stages; ++s) { mbar_init(cfull0 + 8 * s, 1); mbar_init(cempty0 + 8 * s, 8); }
        mbar_init(accf, 1);
        fence_mbar_init();
        tma_prefetch_desc(&map_codes);
        tma_prefetch_desc(&map_x);
    }
    if (warp == 1) { tmem_alloc(smem_u32(&tmem_base_sh), p.tmem_cols); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = tmem_base_sh;
    volatile int* abort_flag = &abort_sh;

    if (warp == 0) {
        uint32_t cs = 0, cph = 1, s = 0, ph = 1;             // parities of the "free" phases to wait for
        bool ok = true;
        for (int kt = kt0; kt < kt1 && ok; ++kt) {
            ok = mbar_wait_uniform(cempty0 + 8 * cs, cph, abort_flag, nullptr);
            if (!ok) break;
            if (elect_one()) {
                const uint32_t bar = cfull0 + 8 * cs, dst = codes0 + cs * ML_CODE_BYTES;
                mbar_expect_tx(bar, ML_CODE_BYTES);
                const long long rt = GRAD ? kt : wt, ct = GRAD ? wt : kt;
                ml_tma_2d(dst, &map_codes, bar, (int)ct * 64, (int)rt * 128);
                bulk_load_1d(dst + 128 * 64, p.scales + (rt * p.pieces + ct) * (long long)MX_SCALE_PIECE, MX_SCALE_PIECE, bar);
            }
            __syncwarp();
            if (++cs == (uint32_t)p.code_stages) { cs = 0; cph ^= 1u; }
            for (int h = 0; h < 2 && ok; ++h) {
                ok = mbar_wait_uniform(empty0 + 8 * s, ph, abort_flag, nullptr);
                if (!ok) break;
                if (elect_one()) {
                    if (p.after && kt == kt0 && h == 0) pdl_wait();
                    mbar_expect_tx(xfull0 + 8 * s, TERMS * term_bytes);
#pragma unroll
                    for (int e = 0; e < TERMS; ++e)          // (rows of a tile past the last token may be another term's: no one stores them)
                        ml_tma_2d(ring0 + s * p.stage_bytes + ML_A_BYTES + e * term_bytes, &map_x, xfull0 + 8 * s, kt * 128 + h * 64, e * p.x_rows + t0);
                }
                __syncwarp();
                if (++s == (uint32_t)p.stages) { s = 0; ph ^= 1u; }
            }
        }
    } else if (warp == 1) {
        const uint32_t idesc = instr_desc_bf16(128, p.o.nt, GRAD ? 1 : 0, 0);
        const uint64_t a0 = GRAD ? smem_desc_sw128(ring0, 8192, 1024) : smem_desc_sw128(ring0, 16, 1024);
        const uint64_t b0 = smem_desc_sw128(ring0 + ML_A_BYTES, 16, 1024);
        const uint64_t astep = GRAD ? 128u : 2u;             // 16 elements of the reduction further, in 16-byte units
        uint32_t s = 0, ph = 0, acc = 0;
        const int lead = TERMS == 1 ? p.o.n_acc : p.o.n_acc - 1;
        bool ok = true;
        for (int i = 0; i < steps && ok; ++i) {
            ok = mbar_wait_uniform(xfull0 + 8 * s, ph, abort_flag, nullptr) && mbar_wait_uniform(afull0 + 8 * s, ph, abort_flag, nullptr);
            if (!ok) break;
            tc_fence_after();
            if (elect_one()) {
                const uint64_t off = (uint64_t)((s * p.stage_bytes) >> 4);
#pragma unroll
                for (int k = 0; k < ML_BK / 16; ++k)
                    umma_bf16(tmem_base + acc * p.o.nt, a0 + off + astep * k, b0 + off + 2 * k, idesc, (i >= lead || k) ? 1u : 0u);
                if constexpr (TERMS == 3) {
                    const uint64_t tb = term_bytes >> 4;
#pragma unroll
                    for (int t = 1; t < 3; ++t)
#pragma unroll
                        for (int k = 0; k < ML_BK / 16; ++k)
                            umma_bf16(tmem_base + lead * p.o.nt, a0 + off + astep * k, b0 + off + t * tb + 2 * k, idesc, (i | k | (t - 1)) ? 1u : 0u);
                }
                umma_commit(empty0 + 8 * s);
            }
            __syncwarp();
            if (++acc == (uint32_t)lead) acc = 0;
            if (++s == (uint32_t)p.stages) { s = 0; ph ^= 1u; }
        }
        if (elect_one()) umma_commit(accf);
        __syncwarp();
    } else {
        constexpr int GROUPS = ML_CONV_WARPS / 4;
        const int g = (warp - 2) >> 2, h = g & 1, t = (threadIdx.x - 64) & 127;
        uint32_t cs = (uint32_t)g >> 1, cph = 0, s = (uint32_t)g, ph = 1;       // (there are at least two pieces and four steps in either ring)
        for (int i = g; i < steps; i += GROUPS) {
            if (!mbar_wait_uniform(cfull0 + 8 * cs, cph, abort_flag, nullptr)) break;
            MlBlocks<GRAD> w;
            w.load(codes0 + cs * ML_CODE_BYTES, t, h, kt0 + (i >> 1), p.red);
            uint32_t o[2][4][4];
            w.convert(o);
            __syncwarp();
            if (lane == 0) mbar_arrive(cempty0 + 8 * cs);
            cs += GROUPS / 2;
            if (cs >= (uint32_t)p.code_stages) { cs -= (uint32_t)p.code_stages; cph ^= 1u; }
            if (!mbar_wait_uniform(empty0 + 8 * s, ph, abort_flag, nullptr)) break;
            w.store(ring0 + s * p.stage_bytes, t, h, o);
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(afull0 + 8 * s);
            s += GROUPS;
            if (s >= (uint32_t)p.stages) { s = (uint32_t)g; ph ^= 1u; }
        }
    }
    mx_finish(p.o, tmem_base, smem, accf, abort_flag, wt, t0, rank, steps, TERMS == 3, [](int, int, float v) { return v; });
    drain_after_abort(abort_flag);
    if (warp == 1) tmem_dealloc(tmem_base, p.tmem_cols);
}

// Tile, split and rings of one call; false when the sizes do not fit the grid.  Tokens to a tile and the split of the reduction
// by a model of a CTA's time in microseconds, times the waves: 2 to begin and end, 0.75 for each piece of W that it converts, and
// per token of its tile 0.02, or 0.035 where the sum goes through the cluster.  (4096 x 4096 in 18.1, 24.6 and 32.5 us with 256
// tokens in one tile and a split of four, 512 in two tiles and two, 512 in four tiles and none: 17, 23 and 29 by the model.)
// Clusters of four and eight do not fill the last SMs of every group of them: 128 in all.
inline bool ml_plan(MlParams& p, bool f32_terms, int sms) {
    const int wts = (int)(((long long)p.o.cols + 127) / 128);
    p.red_tiles = (int)(((long long)p.red + 127) / 128);
    double best = 0;
    for (int cap = f32_terms ? 64 : p.o.y_f32 ? 128 : 256; cap >= 64; cap /= 2) {
        const int tiles = (p.o.M + cap - 1) / cap, nt = ((p.o.M + tiles - 1) / tiles + 15) / 16 * 16;
        const int n_acc = f32_terms ? 5 : 512 / nt < 4 ? 512 / nt : 4, lead = f32_terms ? n_acc - 1 : n_acc;
        const long long ctas = (long long)wts * ((p.o.M + nt - 1) / nt);
        for (int split = 1; split <= 8 && split <= p.red_tiles; split *= 2) {
            // the additions into an accumulator, as far as splitting goes
            const bool more = split < 8 && split * 2 <= p.red_tiles;
            if (more && (long long)p.red_tiles * 8 > (long long)(p.o.y_f32 ? MX_ADDS_F32 : MX_ADDS_BF16) * lead * split) continue;
            const int at_once = split == 1 ? sms : split == 2 ? sms - 4 : sms * 7 / 8;
            const double waves = (double)((ctas * split + at_once - 1) / at_once);
            const double cost = waves * (2 + 0.75 * ((p.red_tiles + split - 1) / split) + nt * (split > 1 ? 0.035 : 0.02));
            if (best == 0 || cost < best) { best = cost; p.o.nt = nt; p.o.split = split; p.o.n_acc = n_acc; }
        }
    }
    const int tok_tiles = (p.o.M + p.o.nt - 1) / p.o.nt;
    p.tmem_cols = 32;
    while (p.tmem_cols < (uint32_t)(p.o.n_acc * p.o.nt)) p.tmem_cols *= 2;
    p.stage_bytes = ML_A_BYTES + (uint32_t)p.o.nt * 128u * (f32_terms ? 3u : 1u);
    p.code_stages = p.o.nt > 128 ? ML_CODES_WIDE : ML_CODES;
    const size_t room = ML_SMEM_MOST - (size_t)p.code_stages * ((ML_CODE_BYTES + 127) / 128 * 128);
    p.stages = (int)(room / p.stage_bytes);
    p.stages = p.stages >= ML_MAX_STAGES ? ML_MAX_STAGES : 4;      // 4 or 8: a group of converters has every fourth
    p.code_at = (uint32_t)p.stages * p.stage_bytes;
    return (long long)wts * p.o.split <= 0x7fffffffLL && tok_tiles <= 65535;
}

}  // namespace pac
