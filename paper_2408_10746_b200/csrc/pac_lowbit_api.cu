// C entries of what a trainer keeps in few bits: the MXFP4 codec and its products, and the AdamW step over a list of
// tensors.  None of them allocates device memory or keeps anything from call to call; all work is enqueued on the
// caller's stream and may be captured.
#include <atomic>
#include <cmath>

#include "pac_adamw_tensors.cuh"
#include "pac_mxfp.cuh"
#include "pac_mxfp_linear.cuh"
#include "pac_mxfp_pair.cuh"
#include "pac_mxfp_product.cuh"
#include "pac_mxfp_product_pair.cuh"

using namespace pac;

namespace {

// Makes `device` current for the length of a call.
struct OnDevice {
    int prev = -1;
    bool ok = false;
    explicit OnDevice(int device) {
        int cur = -1;
        if (cudaGetDevice(&cur) != cudaSuccess) { cudaGetLastError(); return; }
        if (cur == device) { ok = true; return; }
        if (cudaSetDevice(device) != cudaSuccess) { cudaGetLastError(); return; }
        prev = cur;
        ok = true;
    }
    ~OnDevice() { if (prev >= 0) cudaSetDevice(prev); }
};

bool aligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
bool dtype_ok(int t) { return t == PAC_F32 || t == PAC_BF16; }
size_t dtype_size(int t) { return t == PAC_F32 ? 4 : 2; }

constexpr int MOST_DEVICES = 64;
int sm_count(int device) {
    static std::atomic<int> known[MOST_DEVICES];
    const bool keep = device >= 0 && device < MOST_DEVICES;
    int n = keep ? known[device].load(std::memory_order_relaxed) : 0;
    if (n > 0) return n;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device) != cudaSuccess || n < 1) { cudaGetLastError(); return 148; }
    if (keep) known[device].store(n, std::memory_order_relaxed);
    return n;
}
pac_status launched() { return cudaGetLastError() == cudaSuccess ? PAC_OK : PAC_ERR_CUDA; }

// [rows][inner] array of `type` elements with a row pitch in bytes, boxes of box_inner x box_rows; elements outside read as 0.
bool map_2d(CUtensorMap* map, CUtensorMapDataType type, const void* base, long long inner, long long rows, long long pitch, int box_inner, int box_rows,
            CUtensorMapSwizzle swizzle) {
    EncodeTiledFn fn = get_encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)inner, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)pitch};
    const cuuint32_t box[2] = {(cuuint32_t)box_inner, (cuuint32_t)box_rows}, ones[2] = {1, 1};
    return fn(map, type, 2, const_cast<void*>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Sizes that every call on an MXFP4 matrix checks: rows and columns, and tile coordinates that fit 32 bits.
bool matrix_ok(const void* codes, const void* scales, long long rows, int cols) {
    return codes && scales && aligned(codes, 16) && aligned(scales, 16) && rows >= 1 && rows <= 0x7fffff00LL && cols >= 1 && cols <= 0x7fffff00;
}

// Opts a kernel in to all the dynamic shared memory it may ever ask for, once per device; `done` is the kernel's own.
struct OptedIn { std::atomic<bool> on[MOST_DEVICES]; };
cudaError_t opt_in(OptedIn& done, const void* kernel, int device) {
    const bool keep = device >= 0 && device < MOST_DEVICES;
    if (keep && done.on[device].load(std::memory_order_acquire)) return cudaSuccess;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(ML_SMEM_MOST + 1024));
    if (e == cudaSuccess && keep) done.on[device].store(true, std::memory_order_release);
    return e;
}

// Attributes of a launch in clusters of `split`; `after`: it may begin while the kernel before it runs (and waits for it).
unsigned launch_attributes(cudaLaunchAttribute* attr, int split, bool after) {
    unsigned n = 0;
    if (split > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = (unsigned)split; attr[n].val.clusterDim.y = 1; attr[n].val.clusterDim.z = 1;
        ++n;
    }
    if (after) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n].val.programmaticStreamSerializationAllowed = 1;
        ++n;
    }
    return n;
}

template <bool GRAD, int TERMS>
cudaError_t launch_linear(int device, cudaStream_t st, const CUtensorMap& codes, const CUtensorMap& x, const MlParams& p) {
    const auto kernel = mxfp_linear_kernel<GRAD, TERMS>;
    static OptedIn done;
    const cudaError_t e = opt_in(done, (const void*)kernel, device);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(((p.o.cols + 127LL) / 128) * p.o.split), (unsigned)((p.o.M + p.o.nt - 1) / p.o.nt));
    cfg.blockDim = dim3(32 * (2 + ML_CONV_WARPS));
    cfg.dynamicSmemBytes = 1024 + p.code_at + (size_t)p.code_stages * ML_CODE_BYTES;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    cfg.attrs = attr;
    cfg.numAttrs = launch_attributes(attr, p.o.split, p.after);
    return cudaLaunchKernelEx(&cfg, kernel, codes, x, p);
}

// y = A B^T on the block-scaled tensor cores; `rows` of A's codes.
cudaError_t launch_product(int device, cudaStream_t st, const unsigned char* a_codes, int rows, const unsigned char* b_codes, int K, MpParams& p) {
    CUtensorMap ma = {}, mb;
    if ((!p.here && !map_2d(&ma, CU_TENSOR_MAP_DATA_TYPE_UINT8, a_codes, mx_row_bytes(K), rows, mx_row_bytes(K), 128, p.o.nt, CU_TENSOR_MAP_SWIZZLE_128B)) ||
        !map_2d(&mb, CU_TENSOR_MAP_DATA_TYPE_UINT8, b_codes, mx_row_bytes(K), p.o.cols, mx_row_bytes(K), 128, 128, CU_TENSOR_MAP_SWIZZLE_128B))
        return cudaErrorInvalidValue;
    static OptedIn done;
    const cudaError_t e = opt_in(done, (const void*)mxfp_product_kernel, device);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(((p.o.cols + 127LL) / 128) * p.o.split), (unsigned)((rows + p.o.nt - 1) / p.o.nt));
    cfg.blockDim = dim3(320);
    cfg.dynamicSmemBytes = mp_smem(p);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    cfg.attrs = attr;
    cfg.numAttrs = launch_attributes(attr, p.o.split, p.after);
    return cudaLaunchKernelEx(&cfg, mxfp_product_kernel, ma, mb, p);
}

// Scales as [row tiles][pieces][128] words, boxes of the two pieces of a K step.
bool map_scales(CUtensorMap* map, const unsigned char* scales, long long rows, int K) {
    EncodeTiledFn fn = get_encode_fn();
    if (!fn) return false;
    const cuuint64_t pieces = (cuuint64_t)mx_col_pieces(K), dims[3] = {128, pieces, (cuuint64_t)((rows + 127) / 128)}, strides[2] = {512, 512 * pieces};
    const cuuint32_t box[3] = {128, 2, 1}, ones[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, const_cast<unsigned char*>(scales), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// The same for many tokens, by pairs of CTAs.
cudaError_t launch_product_pair(int device, cudaStream_t st, const unsigned char* a_codes, const unsigned char* a_scales, const unsigned char* b_codes,
                                const unsigned char* b_scales, int K, const MqParams& p, int sms) {
    CUtensorMap mx, mw, mxs, mws;
    const long long row = mx_row_bytes(K);
    if (!map_2d(&mx, CU_TENSOR_MAP_DATA_TYPE_UINT8, a_codes, row, p.M, row, 128, 128, CU_TENSOR_MAP_SWIZZLE_128B) ||
        !map_2d(&mw, CU_TENSOR_MAP_DATA_TYPE_UINT8, b_codes, row, p.cols, row, 128, 128, CU_TENSOR_MAP_SWIZZLE_128B) ||
        !map_scales(&mxs, a_scales, p.M, K) || !map_scales(&mws, b_scales, p.cols, K))
        return cudaErrorInvalidValue;
    static OptedIn done;
    const cudaError_t e = opt_in(done, (const void*)mxfp_product_pair_kernel, device);
    if (e != cudaSuccess) return e;
    const long long units = (long long)p.w_units * p.t_units;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2u * (unsigned)(units < sms / 2 ? units : sms / 2));
    cfg.blockDim = dim3(MQ_THREADS);
    cfg.dynamicSmemBytes = MQ_SMEM;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, mxfp_product_pair_kernel, mx, mw, mxs, mws, p);
}

// A few tokens as sums of matrices in MXFP4 (split_mxfp_kernel), then one block-scaled product.
cudaError_t few_tokens(int device, cudaStream_t st, const void* x, int x_dtype, int M, long long ldx, const unsigned char* codes, const unsigned char* scales,
                       int N, int K, void* y, int y_dtype, long long ldy, unsigned char* space) {
    const MsSpace w = ms_space(M, K);
    MpParams p = {};
    p.a_scales = space + w.scales; p.b_scales = scales; p.b_codes = codes;
    p.x = x; p.ldx = ldx; p.x_f32 = x_dtype == PAC_F32; p.K = K;
    p.here = ms_here(M, N, K);
    p.after = !p.here;
    p.o.y = y; p.o.ldy = ldy; p.o.y_f32 = y_dtype == PAC_F32; p.o.M = M; p.o.cols = N; p.o.terms = MS_TERMS;
    p.pieces = mx_col_pieces(K);
    if (!mp_plan(p, K, sm_count(device))) return cudaErrorInvalidValue;
    if (p.here) return launch_product(device, st, nullptr, M * MS_TERMS, codes, K, p);
    const unsigned grid = (unsigned)(((long long)M * p.pieces * 4 + 7) / 8);
    if (x_dtype == PAC_F32) split_mxfp_kernel<float><<<grid, 256, 0, st>>>((const float*)x, M, K, ldx, space + w.codes, space + w.scales);
    else split_mxfp_kernel<bf16><<<grid, 256, 0, st>>>((const bf16*)x, M, K, ldx, space + w.codes, space + w.scales);
    const cudaError_t e = cudaGetLastError();
    return e != cudaSuccess ? e : launch_product(device, st, space + w.codes, M * MS_TERMS, codes, K, p);
}

// Many tokens: pairs of CTAs (pac_mxfp_pair.cuh).  x in bf16, its rows on 16-byte boundaries.
template <bool GRAD>
cudaError_t launch_pair(int device, cudaStream_t st, const CUtensorMap& codes, const CUtensorMap& x, const MrParams& p, int sms) {
    const auto kernel = mxfp_linear_pair_kernel<GRAD>;
    static OptedIn done;
    const cudaError_t e = opt_in(done, (const void*)kernel, device);
    if (e != cudaSuccess) return e;
    const long long units = (long long)p.w_units * p.t_units;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2u * (unsigned)(units < sms / 2 ? units : sms / 2));
    cfg.blockDim = dim3(MR_THREADS);
    cfg.dynamicSmemBytes = MR_SMEM;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, codes, x, p);
}

// Terms of x instead of converting W, up to 16 tokens (twelve times 16 rows are what two CTAs on an SM have room for): always where
// they are made in the product's kernel, else from 4 M values of W on.  16 tokens: 10.8 us against 12 at 4096 x 4096, 20 against 52 at
// 32000 x 4096; at 1000 x 770 8.4 against 7.6, and two launches to pay for instead of one.
bool few(bool grad, int M, int N, int K) { return !grad && M <= MS_MOST_TOKENS && (ms_here(M, N, K) || (long long)N * K >= (4LL << 20)); }
// Steps to each of as few equal parts as have at most `most`.
int equal_part(long long steps, int most) {
    const long long parts = (steps + most - 1) / most;
    return (int)((steps + parts - 1) / parts);
}
// Rows that TMA boxes can read as they are.
bool boxes(const void* x, int dtype, long long ldx) { return dtype == PAC_BF16 && aligned(x, 16) && ldx % 8 == 0; }
long long linear_space(bool grad, const void* x, int dtype, int M, long long ldx, int N, int K) {
    if (few(grad, M, N, K)) return ms_here(M, N, K) ? 0 : ms_space(M, K).bytes;
    const int red = grad ? N : K;
    return boxes(x, dtype, ldx) ? 0 : (dtype == PAC_F32 ? 6LL : 2LL) * M * pack_columns(red);
}

pac_status mxfp_linear(bool grad, int device, void* stream, const void* x, int x_dtype, int M, long long ldx, const unsigned char* codes,
                       const unsigned char* scales, int N, int K, void* y, int y_dtype, long long ldy, void* space, long long space_bytes) {
    const int red = grad ? N : K, out_cols = grad ? K : N;
    if (M < 0 || !matrix_ok(codes, scales, N, K) || !dtype_ok(x_dtype) || !dtype_ok(y_dtype)) return PAC_ERR_INVALID_ARG;
    if (M == 0) return PAC_OK;
    if (!x || !y || ldx < red || ldy < out_cols || M > 0x0fffff00) return PAC_ERR_INVALID_ARG;
    if (!aligned(x, dtype_size(x_dtype)) || !aligned(y, dtype_size(y_dtype))) return PAC_ERR_INVALID_ARG;
    const long long need = linear_space(grad, x, x_dtype, M, ldx, N, K);
    if (need > 0 && (!space || !aligned(space, 256) || space_bytes < need)) return PAC_ERR_INVALID_ARG;
    OnDevice on(device);
    if (!on.ok) return PAC_ERR_CUDA;
    cudaStream_t st = (cudaStream_t)stream;
    auto status = [](cudaError_t e) {
        if (e == cudaSuccess) return PAC_OK;
        cudaGetLastError();
        return PAC_ERR_CUDA;
    };
    if (few(grad, M, N, K)) return status(few_tokens(device, st, x, x_dtype, M, ldx, codes, scales, N, K, y, y_dtype, ldy, (unsigned char*)space));
    const int sms = sm_count(device), terms = x_dtype == PAC_F32 ? 3 : 1;
    const bool y_f32 = y_dtype == PAC_F32;
    long long x_cols = red, x_pitch = ldx;
    if (need > 0) {
        x_cols = x_pitch = pack_columns(red);
        const long long want = ((long long)M * x_cols / 8 + 255) / 256, most = (long long)sms * 32;
        const unsigned grid = (unsigned)(want < most ? want : most);
        const bool vec = aligned(x, 16) && ldx % 4 == 0;
        if (x_dtype == PAC_F32) pack_tokens_kernel<float><<<grid, 256, 0, st>>>((const float*)x, M, red, ldx, vec, (bf16*)space);
        else pack_tokens_kernel<bf16><<<grid, 256, 0, st>>>((const bf16*)x, M, red, ldx, vec, (bf16*)space);
        if (cudaGetLastError() != cudaSuccess) return PAC_ERR_CUDA;
        x = space;
    }
    CUtensorMap mc, mx;
    if (!map_2d(&mc, CU_TENSOR_MAP_DATA_TYPE_UINT8, codes, mx_row_bytes(K), N, mx_row_bytes(K), 64, 128, CU_TENSOR_MAP_SWIZZLE_64B)) return PAC_ERR_CUDA;
    auto map_x = [&](int box_rows) {
        return map_2d(&mx, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, x, x_cols, (long long)terms * M, x_pitch * 2, ML_BK, box_rows, CU_TENSOR_MAP_SWIZZLE_128B);
    };
    const long long w_tiles = (out_cols + 127LL) / 128, units = (w_tiles + 1) / 2 * ((M + 255LL) / 256);
    // pairs where their tiles fill more than half of the SMs (4096 x 4096: 512 tokens, 32 tiles, 33 us in pairs and 25 in tiles of one CTA
    // with a split reduction; 1024 tokens, 64 tiles, 34 either way, 34 and 58 with fp32 results); fp32 results up to where two accumulators take
    // MX_ADDS_F32 additions each (of an fp32 x's first term: see pac_mxfp_pair.cuh)
    if (M > 128 && units * 4 > sms && units <= 0x7fffffffLL && (!y_f32 || red <= 2 * 16 * MX_ADDS_F32)) {
        MrParams r = {};
        r.y = y; r.ldy = ldy; r.y_f32 = y_f32; r.scales = scales;
        r.M = M; r.cols = out_cols; r.red = red; r.pieces = mx_col_pieces(K); r.red_tiles = (int)((red + 127LL) / 128);
        r.w_tiles = (int)w_tiles; r.w_units = (int)((w_tiles + 1) / 2); r.t_units = (int)((M + 255LL) / 256);
        r.n_acc = y_f32 ? 2 : 1;
        r.terms = terms; r.x_rows = M;
        r.part = y_f32 ? 2 * terms * r.red_tiles : equal_part(2LL * terms * r.red_tiles, MX_ADDS_BF16 / 4);
        if (!map_x(128)) return PAC_ERR_CUDA;
        return status(grad ? launch_pair<true>(device, st, mc, mx, r, sms) : launch_pair<false>(device, st, mc, mx, r, sms));
    }
    MlParams p = {};
    p.o.terms = 1;
    p.scales = scales; p.o.y = y; p.o.ldy = ldy; p.o.y_f32 = y_f32;
    p.o.M = M; p.o.cols = out_cols; p.red = red; p.pieces = mx_col_pieces(K); p.x_rows = M;
    p.after = need > 0;
    if (!ml_plan(p, terms == 3, sms)) return PAC_ERR_UNSUPPORTED;
    if (!map_x(p.o.nt)) return PAC_ERR_CUDA;
    if (grad) return status(terms == 3 ? launch_linear<true, 3>(device, st, mc, mx, p) : launch_linear<true, 1>(device, st, mc, mx, p));
    return status(terms == 3 ? launch_linear<false, 3>(device, st, mc, mx, p) : launch_linear<false, 1>(device, st, mc, mx, p));
}

}  // namespace

extern "C" pac_status pac_quantize_mxfp(int device, void* cuda_stream, const void* dev_x, int dtype, long long rows, int cols, long long ldx,
                                        unsigned char* dev_codes, unsigned char* dev_scales) {
    if (rows < 0 || !dtype_ok(dtype) || cols < 1) return PAC_ERR_INVALID_ARG;
    if (rows == 0) return PAC_OK;
    if (!dev_x || !aligned(dev_x, dtype_size(dtype)) || ldx < cols || !matrix_ok(dev_codes, dev_scales, rows, cols)) return PAC_ERR_INVALID_ARG;
    OnDevice on(device);
    if (!on.ok) return PAC_ERR_CUDA;
    const bool vec = aligned(dev_x, 32) && (ldx * (long long)dtype_size(dtype)) % 32 == 0;
    const long long items = (rows + MX_TILE - 1) / MX_TILE * (MX_TILE / 4) * (mx_col_pieces(cols) / 2);
    const long long want = (items + 7) / 8, most = sm_count(device) * 32LL;
    const unsigned grid = (unsigned)(want < most ? want : most);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const MxDiv by_pairs(mx_col_pieces(cols) / 2, items);
    if (dtype == PAC_F32) quantize_mxfp_kernel<float><<<grid, 256, 0, st>>>((const float*)dev_x, rows, cols, ldx, vec, dev_codes, dev_scales, by_pairs);
    else quantize_mxfp_kernel<bf16><<<grid, 256, 0, st>>>((const bf16*)dev_x, rows, cols, ldx, vec, dev_codes, dev_scales, by_pairs);
    return launched();
}

extern "C" pac_status pac_dequantize_mxfp(int device, void* cuda_stream, const unsigned char* dev_codes, const unsigned char* dev_scales, long long rows,
                                          int cols, void* dev_out, int dtype, long long ldo) {
    if (rows < 0 || !dtype_ok(dtype) || cols < 1) return PAC_ERR_INVALID_ARG;
    if (rows == 0) return PAC_OK;
    if (!dev_out || !aligned(dev_out, dtype_size(dtype)) || ldo < cols || !matrix_ok(dev_codes, dev_scales, rows, cols)) return PAC_ERR_INVALID_ARG;
    OnDevice on(device);
    if (!on.ok) return PAC_ERR_CUDA;
    const bool vec = aligned(dev_out, 32) && (ldo * (long long)dtype_size(dtype)) % 32 == 0;
    const long long per_row = mx_row_bytes(cols) / (vec ? 8 : 1), items = rows * per_row;
    const long long want = (items + 255) / 256, most = sm_count(device) * 32LL;
    const unsigned grid = (unsigned)(want < most ? want : most);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const MxDiv by_row(per_row, items);
    if (vec) {
        if (dtype == PAC_F32) dequantize_mxfp_kernel<float><<<grid, 256, 0, st>>>(dev_codes, dev_scales, rows, cols, (float*)dev_out, ldo, by_row);
        else dequantize_mxfp_kernel<bf16><<<grid, 256, 0, st>>>(dev_codes, dev_scales, rows, cols, (bf16*)dev_out, ldo, by_row);
    } else {
        if (dtype == PAC_F32) dequantize_mxfp_any_kernel<float><<<grid, 256, 0, st>>>(dev_codes, dev_scales, rows, cols, (float*)dev_out, ldo, by_row);
        else dequantize_mxfp_any_kernel<bf16><<<grid, 256, 0, st>>>(dev_codes, dev_scales, rows, cols, (bf16*)dev_out, ldo, by_row);
    }
    return launched();
}

extern "C" pac_status pac_mxfp_linear(int device, void* cuda_stream, const void* dev_x, int x_dtype, int M, long long ldx, const unsigned char* dev_codes,
                                      const unsigned char* dev_scales, int N, int K, void* dev_y, int y_dtype, long long ldy, void* dev_workspace,
                                      long long workspace_bytes) {
    return mxfp_linear(false, device, cuda_stream, dev_x, x_dtype, M, ldx, dev_codes, dev_scales, N, K, dev_y, y_dtype, ldy, dev_workspace, workspace_bytes);
}

extern "C" long long pac_mxfp_linear_workspace(const void* dev_x, int x_dtype, int M, long long ldx, int N, int K, int grad) {
    if (M < 1 || M > 0x0fffff00 || N < 1 || N > 0x7fffff00 || K < 1 || K > 0x7fffff00 || !dtype_ok(x_dtype)) return 0;
    return linear_space(grad != 0, dev_x, x_dtype, M, ldx, N, K);
}

extern "C" pac_status pac_mxfp_linear_grad(int device, void* cuda_stream, const void* dev_dy, int dy_dtype, int M, long long lddy,
                                           const unsigned char* dev_codes, const unsigned char* dev_scales, int N, int K, void* dev_dx, int dx_dtype,
                                           long long lddx, void* dev_workspace, long long workspace_bytes) {
    return mxfp_linear(true, device, cuda_stream, dev_dy, dy_dtype, M, lddy, dev_codes, dev_scales, N, K, dev_dx, dx_dtype, lddx, dev_workspace, workspace_bytes);
}

extern "C" pac_status pac_mxfp_product(int device, void* cuda_stream, const unsigned char* dev_a_codes, const unsigned char* dev_a_scales, int M,
                                       const unsigned char* dev_b_codes, const unsigned char* dev_b_scales, int N, int K, void* dev_y, int y_dtype,
                                       long long ldy) {
    if (M < 0 || !matrix_ok(dev_b_codes, dev_b_scales, N, K) || !dtype_ok(y_dtype)) return PAC_ERR_INVALID_ARG;
    if (M == 0) return PAC_OK;
    if (!matrix_ok(dev_a_codes, dev_a_scales, M, K) || !dev_y || !aligned(dev_y, dtype_size(y_dtype)) || ldy < N) return PAC_ERR_INVALID_ARG;
    OnDevice on(device);
    if (!on.ok) return PAC_ERR_CUDA;
    const int sms = sm_count(device);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    cudaError_t e;
    const long long units = (N + 255LL) / 256 * ((M + 255LL) / 256);
    // pairs where their tiles fill more than half of the SMs (4096 x 4096: 512 tokens 12 us either way, 2048 tokens 19 in pairs and 26 in
    // tiles of one CTA); fp32 results up to MX_ADDS_F32 additions into its accumulator
    if (M > 128 && units * 4 > sms && units <= 0x7fffffffLL && (y_dtype != PAC_F32 || K <= 64 * MX_ADDS_F32)) {
        MqParams q = {};
        q.y = dev_y; q.ldy = ldy; q.y_f32 = y_dtype == PAC_F32; q.M = M; q.cols = N; q.steps = (int)((K + 255LL) / 256);
        q.w_units = (int)((N + 255LL) / 256); q.t_units = (int)((M + 255LL) / 256);
        q.part = y_dtype == PAC_F32 ? q.steps : equal_part(q.steps, MX_ADDS_BF16 / 4);
        e = launch_product_pair(device, st, dev_a_codes, dev_a_scales, dev_b_codes, dev_b_scales, K, q, sms);
        if (e == cudaSuccess) return PAC_OK;
        cudaGetLastError();
        return PAC_ERR_CUDA;
    }
    MpParams p = {};
    p.a_scales = dev_a_scales; p.b_scales = dev_b_scales;
    p.o.y = dev_y; p.o.ldy = ldy; p.o.y_f32 = y_dtype == PAC_F32; p.o.M = M; p.o.cols = N;
    p.pieces = mx_col_pieces(K);
    p.o.terms = 1;
    if (!mp_plan(p, K, sms)) return PAC_ERR_UNSUPPORTED;
    e = launch_product(device, st, dev_a_codes, M, dev_b_codes, K, p);
    if (e == cudaSuccess) return PAC_OK;
    cudaGetLastError();
    return PAC_ERR_CUDA;
}

// ---------------------------------------------------------------------------
// AdamW over a list of tensors
// ---------------------------------------------------------------------------
namespace {

unsigned long long blocks_of(const pac_adamw_tensor& t) { return (unsigned long long)((t.n + AT_BLOCK - 1) / AT_BLOCK); }

template <int BITS, int CAP, bool TINY>
cudaError_t launch_adamw(cudaStream_t st, const pac_adamw_tensor* t, int count, AtStep s, int sms) {
    AtList<CAP> list;
    unsigned long long blocks = 0, chunks = 0;
    for (int i = 0; i < count; ++i) blocks += blocks_of(t[i]);
    // a chunk is what one warp takes at a time (its next block is on the way while one is computed): one wave of warps where 16
    // blocks or fewer to each are enough (8.65 M fp32 elements: 33 us at four blocks, in 2.4 waves)
    const unsigned long long resident = (unsigned long long)sms * 24, per = (blocks + resident - 1) / resident;
    s.chunk = per < 1 ? 1u : per > 16 ? 16u : (uint32_t)per;
    for (int i = 0; i < count; ++i) {
        AtTensor& a = list.t[i];
        a.p = t[i].p; a.g = t[i].g; a.m = t[i].m; a.v = t[i].v; a.m_scale = t[i].m_scale; a.v_scale = t[i].v_scale; a.n = t[i].n;
        a.first_chunk = (uint32_t)chunks;
        const size_t pa = t[i].p_dtype == PAC_F32 ? 32 : 16, ga = t[i].g_dtype == PAC_F32 ? 32 : 16, sa = BITS == 32 ? 32 : 8;
        const bool vec = aligned(a.p, pa) && aligned(a.g, ga) && aligned(a.m, sa) && aligned(a.v, sa);
        a.flags = (t[i].p_dtype == PAC_BF16 ? AT_P16 : 0u) | (t[i].g_dtype == PAC_BF16 ? AT_G16 : 0u) | (t[i].decay ? AT_DECAY : 0u) | (vec ? AT_VEC : 0u);
        chunks += (blocks_of(t[i]) + s.chunk - 1) / s.chunk;
    }
    s.count = count;
    s.chunks = (uint32_t)chunks;
    const unsigned long long want = (chunks + 7) / 8, most = (unsigned long long)sms * 32;
    adamw_tensors_kernel<BITS, CAP, TINY><<<(unsigned)(want < most ? want : most), 256, 0, st>>>(list, s);
    return cudaGetLastError();
}
template <int BITS, bool TINY>
cudaError_t launch_list(cudaStream_t st, const pac_adamw_tensor* t, int count, const AtStep& s, int sms) {
    return count <= AT_SMALL ? launch_adamw<BITS, AT_SMALL, TINY>(st, t, count, s, sms) : launch_adamw<BITS, AT_LARGE, TINY>(st, t, count, s, sms);
}

}  // namespace

extern "C" pac_status pac_adamw_tensors(int device, void* cuda_stream, const pac_adamw_tensor* tensors, int count, int state_bits, const pac_adamw* hp,
                                        long long step, const long long* dev_step, float grad_scale, unsigned seed) {
    if (count < 0 || !hp || (state_bits != 8 && state_bits != 32) || (count > 0 && !tensors) || (dev_step ? !aligned(dev_step, 8) : step < 1))
        return PAC_ERR_INVALID_ARG;
    for (int i = 0; i < count; ++i) {
        const pac_adamw_tensor& t = tensors[i];
        if (t.n < 0 || t.n > (1LL << 39) || !dtype_ok(t.p_dtype) || !dtype_ok(t.g_dtype)) return PAC_ERR_INVALID_ARG;
        if (t.n == 0) continue;
        if (!t.p || !t.g || !t.m || !t.v || !aligned(t.p, dtype_size(t.p_dtype)) || !aligned(t.g, dtype_size(t.g_dtype))) return PAC_ERR_INVALID_ARG;
        if (state_bits == 32 && (!aligned(t.m, 4) || !aligned(t.v, 4))) return PAC_ERR_INVALID_ARG;
        if (state_bits == 8 && (!t.m_scale || !t.v_scale || !aligned(t.m_scale, 4) || !aligned(t.v_scale, 4))) return PAC_ERR_INVALID_ARG;
    }
    OnDevice on(device);
    if (!on.ok) return PAC_ERR_CUDA;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (!dev_step) {
        // a replayed graph would take this very step again and again
        cudaStreamCaptureStatus cap = cudaStreamCaptureStatusNone;
        if (cudaStreamIsCapturing(st, &cap) != cudaSuccess) { cudaGetLastError(); return PAC_ERR_CUDA; }
        if (cap != cudaStreamCaptureStatusNone) return PAC_ERR_BAD_STATE;
    }
    AtStep s = {};
    s.hp = *hp; s.grad_scale = grad_scale; s.seed = seed; s.dev_step = dev_step;
    if (!dev_step) {
        s.step = (uint32_t)step;
        s.bc1 = (float)(1.0 - std::pow((double)hp->beta1, (double)step));
        s.bc2 = (float)(1.0 - std::pow((double)hp->beta2, (double)step));
    }
    const int sms = sm_count(device);
    const bool tiny = !((double)hp->eps * std::sqrt(1.0 - (double)hp->beta2) >= 3.637978807091713e-12);      // 2^(25 - 63); bc2 >= 1 - beta2
    for (int at = 0; at < count;) {
        // as many tensors as a list holds and whose blocks a 32-bit number counts; empty tensors only end a run
        int n = 0;
        unsigned long long blocks = 0;
        while (at < count && tensors[at].n == 0) ++at;
        const int most = count - at <= AT_SMALL ? AT_SMALL : AT_LARGE;
        while (at + n < count && n < most && tensors[at + n].n > 0) {
            const unsigned long long b = blocks_of(tensors[at + n]);
            if (blocks + b > 0x7fffffffULL && n > 0) break;
            blocks += b;
            ++n;
        }
        if (n == 0) break;
        s.first_tensor = at;
        const cudaError_t e = state_bits == 32 ? launch_list<32, false>(st, tensors + at, n, s, sms)
                              : tiny           ? launch_list<8, true>(st, tensors + at, n, s, sms)
                                               : launch_list<8, false>(st, tensors + at, n, s, sms);
        if (e != cudaSuccess) return PAC_ERR_CUDA;
        at += n;
    }
    return PAC_OK;
}
