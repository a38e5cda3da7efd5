// Host side of sparq_wgrad_mx8: validation, choice of form, launch.
#include "sparq_wgrad_kernel.cuh"

namespace sparq {

namespace {

// attr_set: per device ordinal, one array for each kernel.
template <class Kernel, class Args>
cudaError_t launch_wgrad(Kernel kernel, bool (&attr_set)[64], int grid, int cluster, int threads, int smem, cudaStream_t st, const CUtensorMap &dy,
                         const CUtensorMap &codes, const CUtensorMap &scales, const Args &args)
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess && (dev < 0 || dev >= 64 || !attr_set[dev])) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e == cudaSuccess && dev >= 0 && dev < 64) attr_set[dev] = true;
    }
    return e == cudaSuccess ? launch_overlapped_cluster(kernel, grid, cluster, threads, smem, st, dy, codes, scales, args) : e;
}

}  // namespace

}  // namespace sparq

using namespace sparq;

extern "C" int sparq_wgrad_mx8(const void *dy, int64_t lddy, const int8_t *codes, const uint8_t *scales,
                               int64_t M, int64_t N, int64_t K, int accumulate, float *dw, void *stream)
{
    if (M < 0 || N < 0 || K < 0) return set_error(SPARQ_ERR_INVALID_ARG, "negative dimension");
    if (N == 0 || K == 0) return SPARQ_OK;
    if (!dw) return set_error(SPARQ_ERR_INVALID_ARG, "dw is NULL");
    if ((uintptr_t)dw & 3u) return set_error(SPARQ_ERR_UNSUPPORTED, "dw must be 4-byte aligned");
    const int64_t most = INT64_C(2147483647) - 255;
    if (M >= most || N >= most || K >= most) return set_error(SPARQ_ERR_UNSUPPORTED, "M, N and K must be below 2^31 - 256");
    cudaStream_t st = (cudaStream_t)stream;
    if (M == 0) {           // a sum over no tokens
        if (accumulate) return SPARQ_OK;
        const cudaError_t e = cudaMemsetAsync(dw, 0, (size_t)N * (size_t)K * sizeof(float), st);
        return e == cudaSuccess ? SPARQ_OK : cuda_error(e, "cudaMemsetAsync(dw)");
    }
    if (!dy || !codes || !scales) return set_error(SPARQ_ERR_INVALID_ARG, "dy/codes/scales pointer is NULL");
    if (M == 1) lddy = round_up64(N, 8);      // a single row has no pitch
    if (lddy < N) return set_error(SPARQ_ERR_INVALID_ARG, "the leading dimension of dy (%lld) is less than N (%lld)", (long long)lddy, (long long)N);
    if (lddy % 8 || ((uintptr_t)dy & 15u)) return set_error(SPARQ_ERR_UNSUPPORTED, "dy must be 16-byte aligned and its leading dimension a multiple of 8");
    if (((uintptr_t)codes | (uintptr_t)scales) & 15u) return set_error(SPARQ_ERR_UNSUPPORTED, "codes and scales must be 16-byte aligned");
    if (lddy > INT64_C(1) << 38) return set_error(SPARQ_ERR_UNSUPPORTED, "the leading dimension of dy is %lld", (long long)lddy);
    int sms = 0, rc = device_info(&sms);
    if (rc != SPARQ_OK) return rc;

    WgradArgs g = {};
    g.M = M;
    g.N = N;
    g.K = K;
    g.blocks = (int)((M + kWgTokens - 1) / kWgTokens);
    g.accumulate = accumulate != 0;
    g.dw = dw;
    g.wait_limit = kWaitLimitCycles;
    if ((rc = get_status_word(&g.status)) != SPARQ_OK) return rc;
    CUtensorMap map_dy, map_codes, map_scales;
    const int64_t pitch = mx_code_pitch(SPARQ_MXINT8, K), spitch = mx_scale_cols(SPARQ_MXINT8, K);
    if ((rc = encode_matrix(&map_dy, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, dy, N, M, lddy * 2, 64, kWgTokens, CU_TENSOR_MAP_SWIZZLE_128B)) != SPARQ_OK) return rc;
    if ((rc = encode_matrix(&map_codes, CU_TENSOR_MAP_DATA_TYPE_UINT8, codes, pitch, M, pitch, kWgBN, kWgTokens, CU_TENSOR_MAP_SWIZZLE_NONE)) != SPARQ_OK) return rc;
    if ((rc = encode_matrix(&map_scales, CU_TENSOR_MAP_DATA_TYPE_UINT8, scales, spitch, M, spitch, 16, kWgTokens, CU_TENSOR_MAP_SWIZZLE_NONE)) != SPARQ_OK) return rc;
    const int64_t n_tiles = (N + kWgTile - 1) / kWgTile, k_tiles = (K + kWgTile - 1) / kWgTile;
    if (n_tiles * k_tiles >= 16 && n_tiles * k_tiles <= INT64_C(1) << 30) {
        const int pairs = (int)(n_tiles * k_tiles < sms / 2 ? n_tiles * k_tiles : sms / 2);
        const WgradPairArgs p = {g, (int)n_tiles, (int)k_tiles, pairs};
        // expanded first, into scratch memory
        const size_t x_bytes = (size_t)M * (size_t)pitch * 2;
        if (n_tiles >= 3) {
            if (void *x = workspace_alloc(x_bytes, st)) {
                CUtensorMap map_x;
                rc = sparq_dequantize_mx(codes, scales, M, K, SPARQ_MXINT8, nullptr, x, SPARQ_DTYPE_BF16, pitch, stream);
                if (rc == SPARQ_OK)
                    rc = encode_matrix(&map_x, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, x, K, M, pitch * 2, 64, kWgTokens, CU_TENSOR_MAP_SWIZZLE_128B);
                if (rc == SPARQ_OK) {
                    static bool set[64] = {};
                    const cudaError_t ce = launch_wgrad(sparq_wgrad_kernel<true>, set, 2 * pairs, 2, kWgPairThreads, wgrad_smem(true), st, map_dy, map_x, map_x, p);
                    if (ce != cudaSuccess) rc = cuda_error(ce, "sparq_wgrad_kernel launch");
                }
                workspace_free(x, st);
                return rc;
            }
        }
        static bool set[64] = {};
        const cudaError_t ce = launch_wgrad(sparq_wgrad_kernel<false>, set, 2 * pairs, 2, kWgPairThreads, wgrad_smem(false), st, map_dy, map_codes, map_scales, p);
        return ce == cudaSuccess ? SPARQ_OK : cuda_error(ce, "sparq_wgrad_kernel launch");
    }
    const int64_t tiles = (N + 127) / 128 * ((K + kWgBN - 1) / kWgBN);
    g.split = 1;
    while (g.split < 8 && tiles <= clusters_at_once(2 * g.split, sms) && g.blocks >= 2 * g.split) g.split *= 2;
    g.stages = kWgStages;
    if (tiles * g.split > INT64_C(2147483647)) return set_error(SPARQ_ERR_UNSUPPORTED, "more than 2^31 tiles");
    static bool set[64] = {};
    const cudaError_t e = launch_wgrad(sparq_wgrad_small_kernel, set, (int)(tiles * g.split), g.split, kWgThreads, wgrad_smem(false), st, map_dy, map_codes, map_scales, g);
    return e == cudaSuccess ? SPARQ_OK : cuda_error(e, "sparq_wgrad_small_kernel launch");
}
