// The product of pac_mxfp_linear.cuh for many tokens: CTAs in pairs (tcgen05.mma.cta_group::2) on tiles of 256 rows of W (or
// columns, backward) x 256 tokens.  Each CTA converts its own 128 rows and brings in half of the tokens, so a code is
// converted once per 256 tokens and a K step of 64 costs an SM 8192 conversions and 20 KB from L2 for 512 clocks of tensor work;
// alone it would be the same conversions and 36 KB.  Persistent pairs; the accumulators of one tile are stored while the
// next tile is computed (bf16 results), or both halves of tensor memory take turns within a tile (fp32 results: half the
// additions into either, counting those of an fp32 x's first term; the other two come first and cut 2^-8 as much).  A reduction of more additions than a bf16 result's accumulator takes is computed in equal parts: one
// half of tensor memory receives a part, the storing warps add it to the sum of the parts before it, which the other half holds.  An fp32 x comes as three bf16 terms and the reduction goes over W three times, the smallest term first: what
// is cut off while the sums are small is smaller still.
//
// Measured: 8192 x 11008 x 4096 in 530 us (1.39 PFLOP/s, 0.99 of the library product's sustained rate), 610 us in runs of tenths of a
// second, where the power cap sets the clock and converting has its share of the power.  With two groups of converting warps
// instead of three 565 us: a group's waits and fences take longer than two steps.
#pragma once
#include "pac_mxfp_linear.cuh"

namespace pac {

constexpr int MR_STAGES = 6, MR_CODES = 3, MR_CONV_WARPS = 12, MR_EPI_WARPS = 4, MR_THREADS = 32 * (2 + MR_CONV_WARPS + MR_EPI_WARPS);
constexpr uint32_t MR_STAGE = 2 * ML_A_BYTES;
constexpr size_t MR_SMEM = 1024 + (size_t)MR_STAGES * MR_STAGE + (size_t)MR_CODES * ML_CODE_BYTES;

struct MrParams {
    void* y; long long ldy; int y_f32;
    const unsigned char* scales;
    int M, cols, red, pieces, red_tiles;
    int w_tiles;                                            // 128-wide tiles of y's columns
    int w_units, t_units;                                   // pairs of them; tiles of 256 tokens
    int n_acc;                                              // accumulators per tile: 1 (two tiles in flight) or 2
    int part;                                               // K steps to a part of the reduction (n_acc 2: all of them)
    int terms, x_rows;                                      // x is the sum of so many matrices of x_rows rows, the last ones (the small ones) first
};

__device__ __forceinline__ void mr_tma_2d(uint32_t dst, const CUtensorMap* map, uint32_t bar_cluster, int c0, int c1) {
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar_cluster), "r"(c0), "r"(c1) : "memory");
}
// An arrival at the pair's first CTA after tiles were written here for its MMAs.  What orders the writes ahead of the MMA's
// reads is the proxy fence before it (the MMA reads this CTA's memory through the asynchronous proxy); no thread there reads
// them, so the arrival needs no release over the cluster, which waits for all of this thread's traffic and made a step of 512
// clocks one of 1300 (8192 x 11008 x 4096: 972 us with it, 568 without).
__device__ __forceinline__ void mr_arrive(uint32_t bar_cluster) { asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar_cluster) : "memory"); }
// The bounded wait of a converged warp, for a barrier at which the pair's other CTA arrives too.
__device__ __forceinline__ bool mr_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
    auto ready = [&] {
        uint32_t ok;
        asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
                     : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
        return ok != 0;
    };
    bool ok = ready();
    if (!ok) {
        const unsigned long long t0 = global_ns();
        for (uint32_t it = 1; !(ok = ready()); ++it)
            if ((it & 63u) == 0 && (*abort_flag || global_ns() - t0 > WAIT_LIMIT_NS)) break;
        if (!ok) *abort_flag = 1;
    }
    return __all_sync(0xffffffffu, ok) != 0;
}

// Warps: 0 copies, 1 MMAs (of the pair's first CTA), 2-13 convert W, 14-17 store y.
template <bool GRAD>
__global__ void __launch_bounds__(MR_THREADS, 1) mxfp_linear_pair_kernel(const __grid_constant__ CUtensorMap map_codes, const __grid_constant__ CUtensorMap map_x,
                                                                         const __grid_constant__ MrParams p) {
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = (unsigned char*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    __shared__ __align__(8) unsigned long long bars[3 * MR_STAGES + 2 * MR_CODES + 4];
    __shared__ uint32_t tmem_base_sh;
    __shared__ int abort_sh;
    const uint32_t xfull0 = smem_u32(&bars[0]), afull0 = smem_u32(&bars[MR_STAGES]), empty0 = smem_u32(&bars[2 * MR_STAGES]);
    const uint32_t cfull0 = smem_u32(&bars[3 * MR_STAGES]), cempty0 = smem_u32(&bars[3 * MR_STAGES + MR_CODES]);
    const uint32_t accf0 = smem_u32(&bars[3 * MR_STAGES + 2 * MR_CODES]), acce0 = accf0 + 16;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cooperative_groups::this_cluster().block_rank();
    const int units = p.w_units * p.t_units, unit0 = (int)(blockIdx.x >> 1), unit_step = (int)(gridDim.x >> 1);
    const uint32_t ring0 = smem_u32(smem), codes0 = ring0 + MR_STAGES * MR_STAGE;

    if (threadIdx.x == 0) {
        abort_sh = 0;
        for (int s = 0; s < MR_STAGES; ++s) { mbar_init(xfull0 + 8 * s, 1); mbar_init(afull0 + 8 * s, 8); mbar_init(empty0 + 8 * s, 1); }
        for (int s = 0; s < MR_CODES; ++s) { mbar_init(cfull0 + 8 * s, 1); mbar_init(cempty0 + 8 * s, 8); }
        for (int b = 0; b < 2; ++b) { mbar_init(accf0 + 8 * b, 1); mbar_init(acce0 + 8 * b, 2 * MR_EPI_WARPS); }
        fence_mbar_init();
        tma_prefetch_desc(&map_codes);
        tma_prefetch_desc(&map_x);
    }
    if (warp == 1) { tmem_alloc_pair(smem_u32(&tmem_base_sh), 512u); tmem_relinquish_pair(); }
    tc_fence_before();
    __syncthreads();
    cooperative_groups::this_cluster().sync();               // the peer's barriers exist before anything arrives at them
    tc_fence_after();
    const uint32_t tmem_base = tmem_base_sh;
    volatile int* abort_flag = &abort_sh;

    if (warp == 0) {
        uint32_t cs = 0, cph = 1, s = 0, ph = 1;
        bool ok = true;
        for (int u = unit0; u < units && ok; u += unit_step) {
            // an odd last tile has no partner: its codes lie outside (zeros), its scales are another tile's, nothing of it is stored
            const int wt = (u % p.w_units) * 2 + (int)rank, t0 = (u / p.w_units) * 256 + (int)rank * 128;
            for (int i = 0, kt = 0, row = t0 + (p.terms - 1) * p.x_rows; i < p.terms * p.red_tiles && ok; ++i) {
                ok = mbar_wait_uniform(cempty0 + 8 * cs, cph, abort_flag, nullptr);
                if (!ok) break;
                if (elect_one()) {
                    const uint32_t bar = cfull0 + 8 * cs, dst = codes0 + cs * ML_CODE_BYTES;
                    mbar_expect_tx(bar, ML_CODE_BYTES);
                    const int rt = GRAD ? kt : wt, ct = GRAD ? wt : kt;
                    ml_tma_2d(dst, &map_codes, bar, ct * 64, rt * 128);
                    const long long piece = (long long)(GRAD ? kt : min(wt, p.w_tiles - 1)) * p.pieces + ct;
                    bulk_load_1d(dst + 128 * 64, p.scales + piece * MX_SCALE_PIECE, MX_SCALE_PIECE, bar);
                }
                __syncwarp();
                if (++cs == MR_CODES) { cs = 0; cph ^= 1u; }
                for (int h = 0; h < 2 && ok; ++h) {
                    ok = mbar_wait_uniform(empty0 + 8 * s, ph, abort_flag, nullptr);
                    if (!ok) break;
                    if (elect_one()) {
                        if (rank == 0) mbar_expect_tx(xfull0 + 8 * s, 2 * ML_A_BYTES);
                        mr_tma_2d(ring0 + s * MR_STAGE + ML_A_BYTES, &map_x, mapa_shared(xfull0 + 8 * s, 0u), kt * 128 + h * 64, row);
                    }
                    __syncwarp();
                    if (++s == MR_STAGES) { s = 0; ph ^= 1u; }
                }
                if (++kt == p.red_tiles) { kt = 0; row -= p.x_rows; }
            }
        }
    } else if (warp == 1) {
        if (rank == 0) {
            const uint32_t idesc = instr_desc_bf16(256, 256, GRAD ? 1 : 0, 0);
            const uint64_t a0 = GRAD ? smem_desc_sw128(ring0, 8192, 1024) : smem_desc_sw128(ring0, 16, 1024);
            const uint64_t b0 = smem_desc_sw128(ring0 + ML_A_BYTES, 16, 1024), astep = GRAD ? 128u : 2u;
            const int steps = 2 * p.terms * p.red_tiles, parts = (steps + p.part - 1) / p.part, n = ((units - unit0 + unit_step - 1) / unit_step) * parts;
            const bool turns = p.n_acc == 1 && parts == 1;   // tiles in both halves of tensor memory by turns
            uint32_t s = 0, ph = 0;
            bool ok = true;
            for (int fill = 0, i0 = 0; fill < n && ok; ++fill) {
                const uint32_t buf = turns ? (uint32_t)fill & 1u : 0u, use = turns ? (uint32_t)fill >> 1 : (uint32_t)fill;
                ok = mr_wait(acce0 + 8 * buf, (use & 1u) ^ 1u, abort_flag);
                if (!ok) break;
                tc_fence_after();
                const int here = min(p.part, steps - i0);
                for (int i = 0; i < here; ++i) {
                    ok = mr_wait(xfull0 + 8 * s, ph, abort_flag) && mr_wait(afull0 + 8 * s, ph, abort_flag);
                    if (!ok) break;
                    tc_fence_after();
                    if (elect_one()) {
                        const uint64_t off = (uint64_t)((s * MR_STAGE) >> 4);
                        const uint32_t d = tmem_base + (p.n_acc == 1 ? buf : (uint32_t)i & 1u) * 256u;
#pragma unroll
                        for (int k = 0; k < ML_BK / 16; ++k)
                            umma_bf16_pair(d, a0 + off + astep * k, b0 + off + 2 * k, idesc, (i >= p.n_acc || k) ? 1u : 0u);
                        umma_commit_pair(empty0 + 8 * s, (uint16_t)3);
                    }
                    __syncwarp();
                    if (++s == MR_STAGES) { s = 0; ph ^= 1u; }
                }
                if (!ok) break;
                if (elect_one()) umma_commit_pair(accf0 + 8 * buf, (uint16_t)3);
                __syncwarp();
                i0 = i0 + here == steps ? 0 : i0 + here;
            }
        }
    } else if (warp < 2 + MR_CONV_WARPS) {
        // three groups of four warps, each with every third step of all this pair's tiles (six stages: its own are two of them)
        constexpr uint32_t GROUPS = MR_CONV_WARPS / 4;
        static_assert(MR_STAGES % GROUPS == 0, "a group's stages are its own");
        // of three pieces a group has a step in two, the same two places of a ring of three every time: it meets those at every
        // fill, and the parities that it waits for are those of the fills it means
        static_assert(MR_CODES == GROUPS && GROUPS == 3, "a group passes over no fill of its places");
        const int g = (warp - 2) >> 2, t = (threadIdx.x - 64) & 127;
        const int steps = 2 * p.terms * p.red_tiles, mine = unit0 < units ? (units - unit0 + unit_step - 1) / unit_step : 0;
        const long long total = (long long)mine * steps;
        uint32_t s = (uint32_t)g, ph = 1, cs = 0, cph = 0;    // cs: ring position of the piece that step n lies in
        int i = g, c = 0;                                    // step within the tile; pieces passed
        const uint32_t afull_first = mapa_shared(afull0, 0u);
        for (long long n = g; n < total; n += GROUPS) {
            for (; c < (int)((n >> 1) & 0x7fffffff); ++c)
                if (++cs == MR_CODES) { cs = 0; cph ^= 1u; }
            while (i >= steps) i -= steps;
            int kt = i >> 1;
            while (kt >= p.red_tiles) kt -= p.red_tiles;
            const int h = i & 1;
            if (!mbar_wait_uniform(cfull0 + 8 * cs, cph, abort_flag, nullptr)) break;
            MlBlocks<GRAD> w;
            w.load(codes0 + cs * ML_CODE_BYTES, t, h, kt, p.red);
            uint32_t o[2][4][4];
            w.convert(o);
            __syncwarp();
            if (lane == 0) mbar_arrive(cempty0 + 8 * cs);
            if (!mbar_wait_uniform(empty0 + 8 * s, ph, abort_flag, nullptr)) break;
            w.store(ring0 + s * MR_STAGE, t, h, o);
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mr_arrive(afull_first + 8 * s);
            s += GROUPS;
            if (s >= MR_STAGES) { s = (uint32_t)g; ph ^= 1u; }
            i += GROUPS;
        }
    } else {
        const int q = warp & 3;
        const uint32_t acce_first = mapa_shared(acce0, 0u), taddr = tmem_base + ((uint32_t)(q * 32) << 16);
        const int steps = 2 * p.terms * p.red_tiles, parts = (steps + p.part - 1) / p.part;
        const bool turns = p.n_acc == 1 && parts == 1;
        uint32_t fill = 0;
        bool ok = true;
        for (int u = unit0; u < units; u += unit_step) {
            const int col = ((u % p.w_units) * 2 + (int)rank) * 128 + q * 32 + lane, t0 = (u / p.w_units) * 256;
            if (parts > 1) {
                // the MMAs wait meanwhile, once in 65000 clocks (2048 tokens, 32000 x 4096: 450-459 us in long runs, 454-497 with all
                // additions in one accumulator); only this warp touches its lanes of the sum
                for (int part = 0; part < parts; ++part, ++fill) {
                    ok = ok && mr_wait(accf0, fill & 1u, abort_flag);
                    tc_fence_after();
#pragma unroll 1
                    for (int c0 = 0; c0 < 256; c0 += 16) {
                        float v[16], w[16];
                        tmem_ld16(taddr + c0, v);
                        if (part) tmem_ld16(taddr + 256u + c0, w);
                        tmem_ld_wait();
                        if (part) {
#pragma unroll
                            for (int e = 0; e < 16; ++e) v[e] += w[e];
                        }
                        tmem_st16(taddr + 256u + c0, v);
                    }
                    tmem_st_wait();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster(acce_first);
                }
            }
            const uint32_t buf = parts > 1 ? 1u : turns ? fill & 1u : 0u;
            if (parts == 1) {
                ok = ok && mr_wait(accf0 + 8 * buf, (turns ? fill >> 1 : fill) & 1u, abort_flag);
                tc_fence_after();
                ++fill;
            }
            const int n_tok = min(256, p.M - t0);
            for (int c0 = 0; c0 < 256; c0 += 16) {
                float v[16], w[16];
                tmem_ld16(taddr + buf * 256u + c0, v);
                if (p.n_acc == 2) tmem_ld16(taddr + 256u + c0, w);
                tmem_ld_wait();
                if (p.n_acc == 2) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) v[e] += w[e];
                }
                if (!ok) {                                   // a wait that ran out leaves NaN, not a wrong number
#pragma unroll
                    for (int e = 0; e < 16; ++e) v[e] = __uint_as_float(0x7fffffffu);
                }
                if (col < p.cols) {
                    if (p.y_f32) mx_store16(static_cast<float*>(p.y) + (long long)(t0 + c0) * p.ldy + col, p.ldy, n_tok - c0, v);
                    else mx_store16(static_cast<bf16*>(p.y) + (long long)(t0 + c0) * p.ldy + col, p.ldy, n_tok - c0, v);
                }
            }
            if (parts > 1) continue;                         // (handed back above)
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(acce_first + 8 * buf);
        }
    }
    tc_fence_before();
    __syncthreads();
    drain_after_abort(abort_flag);
    cooperative_groups::this_cluster().sync();               // neither CTA frees TMEM or leaves while the pair's MMAs or arrivals may still touch it
    if (warp == 1) tmem_dealloc_pair(tmem_base, 512u);
}

}  // namespace pac
