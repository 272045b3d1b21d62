// Product of two matrices in MXFP4 (pac_mxfp.cuh): y = A B^T, A [M][K] tokens, B [N][K] a frozen matrix.
//
// tcgen05.mma kind::mxf4 multiplies packed codes and applies both operands' scales itself: K steps of 64 values, fp32
// accumulators, four times the bf16 rate.  Codes and scales go from memory to shared memory as they are (TMA boxes of 128
// bytes of a row = 256 values; bulk copies of the scales' pieces), tcgen05.cp spreads a piece over tensor memory (row r:
// lane r % 32 of every quadrant, column r / 32, four scales to a 32-bit word), and no thread touches an operand.  As in
// pac_mxfp_linear.cuh the frozen matrix is the M operand and the tokens are the N operand.
//
// What bounds it: up to 64 tokens the bytes of B (32000 x 4096: 12 us, floor 10.7), below some 10 MB of them the latency of one
// CTA from set-up to stores (4096 x 4096: 7 us).  Up to 192 rows of A two CTAs share an SM, so that one's ring fills while the
// other stores; 250 CTAs are then one wave.  (Two tiles of B to a CTA that share the copies of A, one CTA to an SM: 26 us for 16 tokens
// through 32000 x 4096 where this takes 24.)  Many tokens: pac_mxfp_product_pair.cuh.
#pragma once
#include "pac_mxfp_linear.cuh"

namespace pac {

constexpr int MP_BK = 256, MP_MAX_STAGES = 8;
constexpr uint32_t MP_W_BYTES = 128 * 128;
constexpr uint32_t MP_SF_COLS = 24;                          // scales in tensor memory: two sets of up to 24 columns behind the accumulators
// Tokens that are not in 4 bits, a few of them (pac_mxfp_linear): as sums of MS_TERMS matrices in MXFP4, see split_mxfp_kernel.
constexpr int MS_TERMS = 12, MS_MOST_TOKENS = 16, MS_HERE = 4;

struct MpParams {
    MxOut o;
    const unsigned char *a_scales, *b_scales;
    int pieces;                                             // pieces of scales per row tile (even)
    int steps;                                              // ceil(K / 256)
    int stages;
    uint32_t x_bytes, stage_bytes;
    uint32_t tmem_cols, sf_col;
    bool after;                                             // launched ahead of the end of the kernel that writes A
    bool here;                                              // one or two tokens: the terms of x are made in this kernel, step by step
    // sums of terms: what a result that is not a number is formed from again
    const void* x; long long ldx; int x_f32; int K;
    const unsigned char* b_codes;
};

// D[tmem] (+)= A B with one scale per 32 values of a row; sf: tensor-memory addresses of the scales.
__device__ __forceinline__ void umma_mxf4(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %6, 0;\n tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
}
// 32 rows of 16 bytes of shared memory -> 32 lanes x 4 columns, the same in all four quadrants.
__device__ __forceinline__ void tmem_copy_scales(uint32_t taddr, uint64_t desc) {
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
// Shared-memory descriptor without a swizzle: groups of 8 rows of 16 bytes, 128 bytes apart.
__device__ __forceinline__ uint64_t smem_desc_plain(uint32_t saddr) {
    return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)(128 >> 4) << 32) | (1ull << 46);
}
// Instruction descriptor, kind::mxf4: A and B E2M1 (bits 7, 10), both K-major, N >> 3 at bit 17, scales UE8M0 (bit 23), M >> 7 at
// bit 27; which half of a word of scales this K step uses (0 or 2): bits 4 (B) and 29 (A).
__device__ __forceinline__ uint32_t instr_desc_mxf4(int M, int N, uint32_t half) {
    return (half << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(N >> 3) << 17) | (1u << 23) | ((uint32_t)(M >> 7) << 27) | (half << 29);
}

// A block of x, a value per lane, as a sum of MS_TERMS blocks in MXFP4: the first is x rounded, each next one is what the ones
// before it leave, rounded with a scale two powers of two finer, 2^-127 at the least.  What a term leaves is at most 2 of its units (of [6, 8), which
// become 6; else at most 1), so it is below 8 of the next one's, and the twelfth leaves at most 2^-23 of the largest of the 32
// (mostly 2^-26; 2^-129 where scales end): bf16 values within 2^14 of each other enter exactly.  With it the products of a few tokens are block-scaled
// products of the codes of W as they are: nothing converts W, whose bytes are the floor.  (Scales from the remainders' own
// largest gain 0.6 bits a term and cost a reduction over the warp in each of the twelve dependent rounds: twice the time.)
// put_codes(term, word): the codes of this lane's eight neighbours (lane / 8); put_scale(term, byte).  Terms 8 .. 11 come with
// lanes 0 .. 3 of the eight.
template <typename PutCodes, typename PutScale>
__device__ __forceinline__ void ms_terms(float r, PutCodes put_codes, PutScale put_scale) {
    const uint32_t lane = threadIdx.x & 31;
    const bool finite = !__any_sync(0xffffffffu, !(fabsf(r) < __uint_as_float(0x7f800000u)));
    if (!finite) r = 0.f;
    const int e0 = (int)(__reduce_max_sync(0xffffffffu, __float_as_uint(r) & 0x7fffffffu) >> 23) - 2;
    uint32_t w[2] = {0u, 0u};                                // term t's code: nibble t % 8 of word t / 8
#pragma unroll
    for (int t = 0; t < MS_TERMS; ++t) {
        const uint32_t s = (uint32_t)max(e0 - 2 * t, 0);
        uint32_t c;
        asm("{\n .reg .b8 b0;\n cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n mov.b32 %0, {b0, b0, b0, b0};\n}"
            : "=r"(c) : "f"(r * __uint_as_float((254u - s) << 23)), "f"(0.f));
        c &= 15u;
        const uint32_t mag = c & 7u;
        const float v = __uint_as_float((mag < 2u ? mag * 0x3f000000u : (mag + 252u) << 22) | (c & 8u) << 28);
        r = fmaf(v, -mx_scale_f32(s), r);                    // exact: both are multiples of r's last bit, and the difference is smaller
        w[t >> 3] |= c << (4 * (t & 7));
    }
    // eight lanes x eight nibbles transposed: lane j of the eight gets the codes of term j
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (uint32_t d = 4; d >= 1; d >>= 1) {
            const uint32_t low = d == 4 ? 0x0000ffffu : d == 2 ? 0x00ff00ffu : 0x0f0f0f0fu;
            const uint32_t other = __shfl_xor_sync(0xffffffffu, w[h], d);
            w[h] = (lane & d) ? (w[h] & ~low) | ((other >> (4 * d)) & low) : (w[h] & low) | ((other & low) << (4 * d));
        }
    const int t = (int)(lane & 7u);
    put_codes(t, w[0]);
    if (t < MS_TERMS - 8) put_codes(t + 8, w[1]);
    if (lane < MS_TERMS) put_scale((int)lane, finite || lane ? (uint32_t)max(e0 - 2 * (int)lane, 0) : 255u);
}
// A block of x with an infinity or a NaN has no terms but a scale that is not a number, so every sum that it enters comes out
// as NaN: such a result is formed value by value from x itself (rare, and slow).
__device__ __noinline__ float ms_redo(const MpParams& p, int m, int col) {
    const unsigned char* codes = p.b_codes + (long long)col * mx_row_bytes(p.K);
    float y = 0.f;
    for (int k = 0; k < p.K; ++k) {
        const uint32_t c = (codes[k >> 1] >> (4 * (k & 1))) & 15u, mag = c & 7u;
        const uint32_t s = p.b_scales[((long long)(col / MX_TILE) * p.pieces + k / MX_TILE) * MX_SCALE_PIECE + mx_scale_at((uint32_t)col % MX_TILE, (uint32_t)(k % MX_TILE) / MX_BLOCK)];
        const float v = (mag < 2u ? 0.5f * (float)mag : __uint_as_float((mag + 252u) << 22)) * mx_scale_f32(s);
        const float x = p.x_f32 ? static_cast<const float*>(p.x)[m * p.ldx + k] : __bfloat162float(static_cast<const bf16*>(p.x)[m * p.ldx + k]);
        y = fmaf(x, c & 8u ? -v : v, y);
    }
    return y;
}

// Warps: 0 copies, 1 scales and MMAs, 2-9 store y.
__global__ void __launch_bounds__(320, 2) mxfp_product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ MpParams p) {
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = (unsigned char*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    __shared__ __align__(8) unsigned long long bars[2 * MP_MAX_STAGES + 1];
    __shared__ uint32_t tmem_base_sh;
    __shared__ int abort_sh;
    const uint32_t full0 = smem_u32(&bars[0]), empty0 = smem_u32(&bars[MP_MAX_STAGES]), accf = smem_u32(&bars[2 * MP_MAX_STAGES]);
    const int warp = threadIdx.x >> 5;
    const int rank = p.o.split > 1 ? (int)(blockIdx.x % p.o.split) : 0;
    const int wt = blockIdx.x / p.o.split, t0 = blockIdx.y * p.o.nt;
    const int k0 = (int)((long long)p.steps * rank / p.o.split), k1 = (int)((long long)p.steps * (rank + 1) / p.o.split);
    const uint32_t ring0 = smem_u32(smem);
    // pieces of scales that the tile's tokens lie in (t0 is a multiple of 128); past the last row there are none
    const int t_tiles = (int)min((long long)(p.o.nt + 127) / 128, ((long long)p.o.M * p.o.terms - t0 + 127) / 128);

    float mine[MS_HERE];                                     // this warp's blocks of x, token by token within a step
#pragma unroll
    for (int i = 0; i < MS_HERE; ++i) {
        const int k = k0 + (p.o.M == 1 ? i : i >> 1), m = p.o.M == 1 ? 0 : i & 1, col = k * MP_BK + (warp - 2) * MX_BLOCK + (int)(threadIdx.x & 31);
        mine[i] = !p.here || warp < 2 || k >= k1 || col >= p.K ? 0.f
                  : p.x_f32 ? static_cast<const float*>(p.x)[m * p.ldx + col] : __bfloat162float(static_cast<const bf16*>(p.x)[m * p.ldx + col]);
    }

    if (threadIdx.x == 0) {
        abort_sh = 0;
        for (int s = 0; s < p.stages; ++s) { mbar_init(full0 + 8 * s, p.here ? 9 : 1); mbar_init(empty0 + 8 * s, 1); }
        mbar_init(accf, 1);
        fence_mbar_init();
        if (!p.here) tma_prefetch_desc(&map_a);
        tma_prefetch_desc(&map_b);
    }
    if (warp == 1) { tmem_alloc(smem_u32(&tmem_base_sh), p.tmem_cols); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = tmem_base_sh;
    volatile int* abort_flag = &abort_sh;
    // a stage: codes of the matrix, codes of the tokens, scales of the matrix (2 pieces), scales of the tokens (2 per 128)
    const uint32_t sf_at = MP_W_BYTES + p.x_bytes;

    if (warp == 0) {
        const uint32_t bytes = MP_W_BYTES + 2 * MX_SCALE_PIECE + (p.here ? 0u : p.x_bytes + 2 * MX_SCALE_PIECE * t_tiles);
        auto load_b = [&](int k, uint32_t s) {
            const uint32_t bar = full0 + 8 * s, dst = ring0 + s * p.stage_bytes;
            mbar_expect_tx(bar, bytes);
            ml_tma_2d(dst, &map_b, bar, k * 128, wt * 128);
            bulk_load_1d(dst + sf_at, p.b_scales + ((long long)wt * p.pieces + 2 * k) * MX_SCALE_PIECE, 2 * MX_SCALE_PIECE, bar);
        };
        auto load_a = [&](int k, uint32_t s) {
            if (p.here) return;
            const uint32_t bar = full0 + 8 * s, dst = ring0 + s * p.stage_bytes;
            ml_tma_2d(dst + MP_W_BYTES, &map_a, bar, k * 128, t0);
            for (int i = 0; i < t_tiles; ++i)
                bulk_load_1d(dst + sf_at + 2 * MX_SCALE_PIECE * (1 + i), p.a_scales + ((long long)(t0 / 128 + i) * p.pieces + 2 * k) * MX_SCALE_PIECE,
                             2 * MX_SCALE_PIECE, bar);
        };
        // the frozen matrix does not wait for the kernel before: its tiles of the first round come in meanwhile
        const int first = min(p.stages, k1 - k0);
        if (elect_one()) {
            for (int i = 0; i < first; ++i) load_b(k0 + i, (uint32_t)i);
            if (p.after) pdl_wait();
            for (int i = 0; i < first; ++i) load_a(k0 + i, (uint32_t)i);
        }
        __syncwarp();
        uint32_t s = 0, ph = 0;
        for (int k = k0 + first; k < k1; ++k) {
            if (!mbar_wait_uniform(empty0 + 8 * s, ph, abort_flag, nullptr)) break;
            if (elect_one()) {
                load_b(k, s);
                load_a(k, s);
            }
            __syncwarp();
            if (++s == (uint32_t)p.stages) { s = 0; ph ^= 1u; }
        }
    } else if (warp == 1) {
        const uint32_t idesc0 = instr_desc_mxf4(128, p.o.nt, 0u), idesc1 = instr_desc_mxf4(128, p.o.nt, 2u);
        const uint64_t w0 = smem_desc_sw128(ring0, 16, 1024), x0 = smem_desc_sw128(ring0 + MP_W_BYTES, 16, 1024), f0 = smem_desc_plain(ring0 + sf_at);
        uint32_t s = 0, ph = 0, acc = 0;
        for (int i = 0; i < k1 - k0; ++i) {
            if (!mbar_wait_uniform(full0 + 8 * s, ph, abort_flag, nullptr)) break;
            tc_fence_after();
            if (elect_one()) {
                const uint64_t off = (uint64_t)((s * p.stage_bytes) >> 4);
                const uint32_t sf = tmem_base + p.sf_col + (i & 1) * MP_SF_COLS;   // copies and MMAs of one thread take effect in order
#pragma unroll
                for (int c = 0; c < 2; ++c) {                // 128 values of K: one word of scales per row
                    tmem_copy_scales(sf + c * 4, f0 + off + c * (MX_SCALE_PIECE >> 4));
                    for (int t = 0; t < t_tiles; ++t)
                        tmem_copy_scales(sf + 8 + c * 8 + t * 4, f0 + off + (2 * (1 + t) + c) * (MX_SCALE_PIECE >> 4));
                }
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    umma_mxf4(tmem_base + acc * p.o.nt, w0 + off + 2 * k, x0 + off + 2 * k, (k & 1) ? idesc1 : idesc0, sf + (k >> 1) * 4, sf + 8 + (k >> 1) * 8,
                              (i >= p.o.n_acc || k) ? 1u : 0u);
                umma_commit(empty0 + 8 * s);
            }
            __syncwarp();
            if (++acc == (uint32_t)p.o.n_acc) acc = 0;
            if (++s == (uint32_t)p.stages) { s = 0; ph ^= 1u; }
        }
        if (elect_one()) umma_commit(accf);
        __syncwarp();
    }
    if (p.here && warp >= 2) {
        // the terms of a step's 256 columns, a block of 32 per warp, where copies would have put them
        const int lane = threadIdx.x & 31, b = warp - 2;
        uint32_t s = 0, ph = 1;
#pragma unroll 1                                                // (once through little code: instructions come from L2 here)
        for (int i = 0; i < MS_HERE; ++i) {
            const int k = k0 + (p.o.M == 1 ? i : i >> 1), m = p.o.M == 1 ? 0 : i & 1;
            if (k >= k1) break;
            const float r = i < 2 ? (i == 0 ? mine[0] : mine[1]) : (i == 2 ? mine[2] : mine[3]);
            if (m == 0 && !mbar_wait_uniform(empty0 + 8 * s, ph, abort_flag, nullptr)) break;
            const uint32_t tile = ring0 + s * p.stage_bytes + MP_W_BYTES, sf = ring0 + s * p.stage_bytes + sf_at + 2 * MX_SCALE_PIECE + (uint32_t)(b >> 2) * MX_SCALE_PIECE;
            ms_terms(r,
                     [&](int t, uint32_t word) {
                         const uint32_t row = (uint32_t)(t * p.o.M + m);
                         asm volatile("st.shared.b32 [%0], %1;" ::"r"(tile + row * 128u + (((uint32_t)b ^ (row & 7u)) << 4) + (uint32_t)(lane >> 3) * 4u), "r"(word) : "memory");
                     },
                     [&](int t, uint32_t scale) { asm volatile("st.shared.u8 [%0], %1;" ::"r"(sf + mx_scale_at((uint32_t)(t * p.o.M + m), (uint32_t)b & 3u)), "r"(scale) : "memory"); });
            if (m + 1 < p.o.M) continue;
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(full0 + 8 * s);
            if (++s == (uint32_t)p.stages) { s = 0; ph ^= 1u; }
        }
    }
    mx_finish(p.o, tmem_base, smem, accf, abort_flag, wt, t0, rank, k1 - k0, false,
              [&](int m, int col, float v) { return p.o.terms > 1 && v != v ? ms_redo(p, m, col) : v; });
    drain_after_abort(abort_flag);
    if (warp == 1) tmem_dealloc(tmem_base, p.tmem_cols);
}

// One or two tokens whose terms are made in the product's own kernel, which saves a launch and the workspace: how many CTAs
// share a reduction (two CTAs on each of B200's 148 SMs; a constant, since the size of the workspace is asked for without naming
// a device), and whether what each has to make is little enough (a step of 256 columns and
// one token is about 1000 clocks of 12 dependent rounds).
constexpr int MS_HERE_CTAS = 296;
inline int ms_here_split(int N, int K) {
    const long long wts = ((long long)N + 127) / 128;
    const int steps = (int)(((long long)K + MP_BK - 1) / MP_BK);
    int split = 1;
    while (split < 8 && split * 2 <= steps && wts * split * 2 <= MS_HERE_CTAS) split *= 2;
    return split;
}
inline bool ms_here(int M, int N, int K) {
    const int steps = (int)(((long long)K + MP_BK - 1) / MP_BK), split = ms_here_split(N, K);
    return M <= 2 && M * ((steps + split - 1) / split) <= MS_HERE;
}

// Sizes and split of a call; terms > 1: A is a sum of so many matrices of o.M rows each, below one another.
inline bool mp_plan(MpParams& p, int K, int sms) {
    const int rows = p.o.M * p.o.terms;
    const long long wts = ((long long)p.o.cols + 127) / 128;
    // 256 tokens to a tile where that gives every SM one (1000 x 4000, 512 tokens: 10 us with 128 to a tile, 22 with 256)
    const int cap = p.o.terms == 1 && (p.o.y_f32 || wts * ((rows + 255LL) / 256) < sms) ? 128 : 256;
    // several token tiles begin at multiples of 128, where the pieces of scales do
    p.o.nt = rows <= cap ? (rows + 15) / 16 * 16 : cap;
    const int tok_tiles = (rows + p.o.nt - 1) / p.o.nt;
    const long long ctas = wts * tok_tiles;
    p.steps = (int)(((long long)K + MP_BK - 1) / MP_BK);
    p.x_bytes = (uint32_t)p.o.nt * 128u;
    p.stage_bytes = MP_W_BYTES + p.x_bytes + 2 * MX_SCALE_PIECE * (uint32_t)(1 + (p.o.nt + 127) / 128);
    p.stage_bytes = (p.stage_bytes + 1023u) / 1024u * 1024u;
    // up to 192 tokens two CTAs share an SM: half the tensor memory and half the shared memory each
    const bool two = p.o.nt <= 192;
    const int acc_cols = two ? 208 : 464;
    p.tmem_cols = two ? 256 : 512;
    p.sf_col = (uint32_t)acc_cols;
    p.o.n_acc = acc_cols / p.o.nt < 3 ? acc_cols / p.o.nt : 3;
    p.o.split = 1;
    if (p.here) p.o.split = ms_here_split(p.o.cols, K);
    while (!p.here && p.o.split < 8 && p.o.split * 2 <= p.steps && ctas * p.o.split * 2 <= sms) p.o.split *= 2;
    // the additions into an accumulator, as far as splitting goes
    while (p.o.split < 8 && p.o.split * 2 <= p.steps && (long long)p.steps * 4 > (long long)(p.o.y_f32 ? MX_ADDS_F32 : MX_ADDS_BF16) * p.o.n_acc * p.o.split) p.o.split *= 2;
    p.stages = (int)((two ? (ML_SMEM_MOST - 4096) / 2 : ML_SMEM_MOST) / p.stage_bytes);
    if (p.stages > MP_MAX_STAGES) p.stages = MP_MAX_STAGES;
    return wts * p.o.split <= 0x7fffffffLL && tok_tiles <= 65535;
}
// Shared memory of a CTA: the ring, and room for partial sums where they go through it.
inline size_t mp_smem(const MpParams& p) {
    const size_t ring = (size_t)p.stages * p.stage_bytes, part = p.o.split > 1 || p.o.terms > 1 ? (size_t)p.o.nt * 512 : 0;
    return 1024 + (ring > part ? ring : part);
}

// x [M][K] in MS_TERMS matrices (ms_terms), term t in rows t M .. t M + M - 1.  A warp takes a block.
template <typename T>
__global__ void __launch_bounds__(256) split_mxfp_kernel(const T* __restrict__ x, int M, int K, long long ldx, unsigned char* __restrict__ codes,
                                                         unsigned char* __restrict__ scales) {
    pdl_trigger();
    const int lane = threadIdx.x & 31, pieces = mx_col_pieces(K), blocks = pieces * 4;
    const long long row_bytes = mx_row_bytes(K);
    const int id = (int)(blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5)), m = id / blocks, b = id - m * blocks;      // (threads may pass 32 bits, warps do not)
    if (m >= M) return;
    const int col = b * MX_BLOCK + lane;
    ms_terms(col < K ? to_f32(x[m * ldx + col]) : 0.f,
             [&](int t, uint32_t word) {
                 if (b * 16 < row_bytes) *reinterpret_cast<uint32_t*>(codes + (t * M + m) * row_bytes + b * 16 + (lane >> 3) * 4) = word;
             },
             [&](int t, uint32_t s) {
                 const int row = t * M + m;
                 scales[((long long)(row / MX_TILE) * pieces + b / 4) * MX_SCALE_PIECE + mx_scale_at((uint32_t)(row % MX_TILE), (uint32_t)b % 4u)] = (unsigned char)s;
             });
}
// The workspace that holds the terms.
struct MsSpace { long long codes, scales, bytes; };
inline MsSpace ms_space(int M, int K) {
    MsSpace w;
    const long long rows = (long long)M * MS_TERMS;
    w.codes = 0;
    w.scales = (rows * mx_row_bytes(K) + 255) / 256 * 256;
    w.bytes = w.scales + (rows + MX_TILE - 1) / MX_TILE * mx_col_pieces(K) * (long long)MX_SCALE_PIECE;
    return w;
}

}  // namespace pac
