// The block-scaled product of pac_mxfp_product.cuh for many tokens: pairs of CTAs (cta_group::2) on tiles of 256 rows of the
// frozen matrix x 256 tokens, persistent.  A K step of 256 values takes 512 clocks of tensor work and brings 35 KB into each SM
// (codes of its own 128 rows and of half of the tokens, scales of its own rows and of all the tokens), close to the 64 bytes per
// clock that an SM receives from L2; a CTA alone brings in 51 KB.  Tensor memory holds one accumulator of 256 columns beside the
// scales, so the eight storing warps take a finished tile into registers at once (128 values a thread) and hand it back before
// they store, while the next tile's copies are already in the ring.  A reduction of more additions than an accumulator takes
// (MX_ADDS_BF16) comes in equal parts, which are added up in those registers.
//
// Measured: 8192 x 11008 x 4096 in some 145 us (5 PFLOP/s; a CTA alone on 128 x 256 tiles, one after another: 315 us).
#pragma once
#include "pac_mxfp_pair.cuh"
#include "pac_mxfp_product.cuh"

namespace pac {

constexpr int MQ_STAGES = 6, MQ_EPI_WARPS = 8, MQ_THREADS = 32 * (2 + MQ_EPI_WARPS);
constexpr uint32_t MQ_W_SF = 2 * 128 * 128, MQ_X_SF = MQ_W_SF + 2 * MX_SCALE_PIECE, MQ_BYTES = MQ_X_SF + 4 * MX_SCALE_PIECE;
constexpr uint32_t MQ_STAGE = (MQ_BYTES + 1023) / 1024 * 1024;
constexpr size_t MQ_SMEM = 1024 + (size_t)MQ_STAGES * MQ_STAGE;
constexpr uint32_t MQ_SF_COL = 256;

struct MqParams {
    void* y; long long ldy; int y_f32;
    int M, cols, steps;                                     // steps of 256 values
    int part;                                               // steps to a part of the reduction
    int w_units, t_units;
};

__device__ __forceinline__ void mq_tma_3d(uint32_t dst, const CUtensorMap* map, uint32_t bar_cluster, int c0, int c1, int c2) {
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar_cluster), "r"(c0), "r"(c1), "r"(c2) : "memory");
}
__device__ __forceinline__ void umma_mxf4_pair(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t sfa, uint32_t sfb, uint32_t accumulate) {
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %6, 0;\n tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate) : "memory");
}
// In both CTAs of the pair, each from its own shared memory.
__device__ __forceinline__ void tmem_copy_scales_pair(uint32_t taddr, uint64_t desc) {
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}

// Warps: 0 copies, 1 scales and MMAs (of the pair's first CTA), 2-9 store y.  map_ws, map_xs: the scales as [row tiles][pieces][128] words.
__global__ void __launch_bounds__(MQ_THREADS, 1)
mxfp_product_pair_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_xs,
                         const __grid_constant__ CUtensorMap map_ws, const __grid_constant__ MqParams p) {
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = (unsigned char*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    __shared__ __align__(8) unsigned long long bars[2 * MQ_STAGES + 2];
    __shared__ uint32_t tmem_base_sh;
    __shared__ int abort_sh;
    const uint32_t full0 = smem_u32(&bars[0]), empty0 = smem_u32(&bars[MQ_STAGES]), accf = smem_u32(&bars[2 * MQ_STAGES]), acce = accf + 8;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cooperative_groups::this_cluster().block_rank();
    const int units = p.w_units * p.t_units, unit0 = (int)(blockIdx.x >> 1), unit_step = (int)(gridDim.x >> 1);
    const uint32_t ring0 = smem_u32(smem);

    if (threadIdx.x == 0) {
        abort_sh = 0;
        for (int s = 0; s < MQ_STAGES; ++s) { mbar_init(full0 + 8 * s, 1); mbar_init(empty0 + 8 * s, 1); }
        mbar_init(accf, 1);
        mbar_init(acce, 2 * MQ_EPI_WARPS);
        fence_mbar_init();
        tma_prefetch_desc(&map_x); tma_prefetch_desc(&map_w); tma_prefetch_desc(&map_xs); tma_prefetch_desc(&map_ws);
    }
    if (warp == 1) { tmem_alloc_pair(smem_u32(&tmem_base_sh), 512u); tmem_relinquish_pair(); }
    tc_fence_before();
    __syncthreads();
    cooperative_groups::this_cluster().sync();               // the peer's barriers exist before anything arrives at them
    tc_fence_after();
    const uint32_t tmem_base = tmem_base_sh;
    volatile int* abort_flag = &abort_sh;

    if (warp == 0) {
        uint32_t s = 0, ph = 1;
        bool ok = true;
        for (int u = unit0; u < units && ok; u += unit_step) {
            const int wt = (u % p.w_units) * 2 + (int)rank, tt = (u / p.w_units) * 2;      // tiles of 128 rows; what lies outside is zeros
            for (int k = 0; k < p.steps; ++k) {
                ok = mbar_wait_uniform(empty0 + 8 * s, ph, abort_flag, nullptr);
                if (!ok) break;
                if (elect_one()) {
                    const uint32_t dst = ring0 + s * MQ_STAGE, bar = mapa_shared(full0 + 8 * s, 0u);
                    if (rank == 0) mbar_expect_tx(full0 + 8 * s, 2 * MQ_BYTES);
                    mr_tma_2d(dst, &map_w, bar, k * 128, wt * 128);
                    mr_tma_2d(dst + MP_W_BYTES, &map_x, bar, k * 128, (tt + (int)rank) * 128);
                    mq_tma_3d(dst + MQ_W_SF, &map_ws, bar, 0, 2 * k, wt);
                    mq_tma_3d(dst + MQ_X_SF, &map_xs, bar, 0, 2 * k, tt);
                    mq_tma_3d(dst + MQ_X_SF + 2 * MX_SCALE_PIECE, &map_xs, bar, 0, 2 * k, tt + 1);
                }
                __syncwarp();
                if (++s == MQ_STAGES) { s = 0; ph ^= 1u; }
            }
        }
    } else if (warp == 1) {
        if (rank == 0) {
            const uint32_t idesc0 = instr_desc_mxf4(256, 256, 0u), idesc1 = instr_desc_mxf4(256, 256, 2u);
            const uint64_t w0 = smem_desc_sw128(ring0, 16, 1024), x0 = smem_desc_sw128(ring0 + MP_W_BYTES, 16, 1024);
            const uint64_t wf0 = smem_desc_plain(ring0 + MQ_W_SF), xf0 = smem_desc_plain(ring0 + MQ_X_SF);
            const int n = ((units - unit0 + unit_step - 1) / unit_step) * ((p.steps + p.part - 1) / p.part);
            uint32_t s = 0, ph = 0, set = 0;
            bool ok = true;
            for (int fill = 0, i0 = 0; fill < n && ok; ++fill) {
                ok = mr_wait(acce, ((uint32_t)fill & 1u) ^ 1u, abort_flag);
                if (!ok) break;
                tc_fence_after();
                const int here = min(p.part, p.steps - i0);
                for (int i = 0; i < here; ++i) {
                    ok = mr_wait(full0 + 8 * s, ph, abort_flag);
                    if (!ok) break;
                    tc_fence_after();
                    if (elect_one()) {
                        const uint64_t off = (uint64_t)((s * MQ_STAGE) >> 4), piece = MX_SCALE_PIECE >> 4;
                        const uint32_t sf = tmem_base + MQ_SF_COL + set * MP_SF_COLS;      // copies and MMAs of one thread take effect in order
#pragma unroll
                        for (int c = 0; c < 2; ++c) {        // 128 values of K: one word of scales per row
                            tmem_copy_scales_pair(sf + c * 4, wf0 + off + c * piece);
                            tmem_copy_scales_pair(sf + 8 + c * 8, xf0 + off + c * piece);
                            tmem_copy_scales_pair(sf + 12 + c * 8, xf0 + off + (2 + c) * piece);
                        }
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            umma_mxf4_pair(tmem_base, w0 + off + 2 * k, x0 + off + 2 * k, (k & 1) ? idesc1 : idesc0, sf + (k >> 1) * 4, sf + 8 + (k >> 1) * 8, (i | k) ? 1u : 0u);
                        umma_commit_pair(empty0 + 8 * s, (uint16_t)3);
                    }
                    __syncwarp();
                    set ^= 1u;
                    if (++s == MQ_STAGES) { s = 0; ph ^= 1u; }
                }
                if (!ok) break;
                if (elect_one()) umma_commit_pair(accf, (uint16_t)3);
                __syncwarp();
                i0 = i0 + here == p.steps ? 0 : i0 + here;
            }
        }
    } else {
        const int q = warp & 3, half = (warp - 2) >> 2;
        const uint32_t acce_first = mapa_shared(acce, 0u), taddr = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)half * 128u;
        uint32_t fill = 0;
        bool ok = true;
        for (int u = unit0; u < units; u += unit_step) {
            const int col = ((u % p.w_units) * 2 + (int)rank) * 128 + q * 32 + lane, t0 = (u / p.w_units) * 256 + half * 128;
            float v[8][16];
            for (int i0 = 0; i0 < p.steps; i0 += p.part, ++fill) {
                ok = ok && mr_wait(accf, fill & 1u, abort_flag);
                tc_fence_after();
                if (i0 == 0) {
#pragma unroll
                    for (int c = 0; c < 8; ++c) tmem_ld16(taddr + c * 16, v[c]);
                    tmem_ld_wait();
                } else {
#pragma unroll
                    for (int c = 0; c < 16; ++c) {
                        float w[8];                          // (what is left of the registers)
                        tmem_ld8(taddr + c * 8, w);
                        tmem_ld_wait();
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[c >> 1][(c & 1) * 8 + e] += w[e];
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(acce_first);
            }
            if (!ok) {                                       // a wait that ran out leaves NaN, not a wrong number
#pragma unroll
                for (int c = 0; c < 128; ++c) v[c >> 4][c & 15] = __uint_as_float(0x7fffffffu);
            }
            if (col < p.cols) {
                const int n_tok = p.M - t0;
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    if (p.y_f32) mx_store16(static_cast<float*>(p.y) + (long long)(t0 + c * 16) * p.ldy + col, p.ldy, n_tok - c * 16, v[c]);
                    else mx_store16(static_cast<bf16*>(p.y) + (long long)(t0 + c * 16) * p.ldy + col, p.ldy, n_tok - c * 16, v[c]);
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    drain_after_abort(abort_flag);
    cooperative_groups::this_cluster().sync();               // neither CTA frees TMEM or leaves while the pair's MMAs or arrivals may still touch it
    if (warp == 1) tmem_dealloc_pair(tmem_base, 512u);
}

}  // namespace pac
