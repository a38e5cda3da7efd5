// Host side of sparq_gemm_mxf4: validation, choice of form, launch.
#include "sparq_mxf4_kernel.cuh"

namespace sparq {

namespace {

constexpr int kMxMaxDynSmem = 232448 - 4096;

template <int BN, bool NV, bool SWAP>
cudaError_t launch_small(const CUtensorMap (&map)[6], MxGemmArgs &g, int64_t grid, cudaStream_t st)
{
    auto kernel = sparq_mxf4_small_kernel<BN, NV, SWAP>;
    static bool attr_set[64] = {};   // per device ordinal
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64 || !attr_set[dev]) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMxMaxDynSmem);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64) attr_set[dev] = true;
    }
    const int64_t C = SWAP ? g.M : g.N;
    const int recv = mx_recv_bytes(mx_own_groups(C < BN ? C : BN, g.split, SWAP), g.split, SWAP), stage = mx_small_stage(BN, NV);
    const int steps = (g.k_blocks + g.split - 1) / g.split, fit = (kMxMaxDynSmem - 1024 - recv) / stage;
    g.stages = steps < fit ? steps : fit;
    if (g.stages > kMaxStages) g.stages = kMaxStages;
    return launch_overlapped_cluster(kernel, (int)grid, g.split, mx_small_threads(SWAP), 1024 + g.stages * stage + recv, st, map[0], map[1], map[4], map[5], g);
}

template <int BN, bool SWAP>
cudaError_t launch_small_of(bool nv, const CUtensorMap (&map)[6], MxGemmArgs &g, int64_t grid, cudaStream_t st)
{
    return nv ? launch_small<BN, true, SWAP>(map, g, grid, st) : launch_small<BN, false, SWAP>(map, g, grid, st);
}

template <bool NV>
cudaError_t launch_pair(const CUtensorMap (&map)[6], const MxPairArgs &p, cudaStream_t st)
{
    auto kernel = sparq_mxf4_kernel<NV>;
    const int smem = pair_smem(NV);
    static bool attr_set[64] = {};   // per device ordinal
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64 || !attr_set[dev]) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64) attr_set[dev] = true;
    }
    return launch_overlapped_cluster(kernel, 2 * p.pairs, 2, kPairThreads, smem, st, map[0], map[1], map[2], map[3], map[4], map[5], p);
}

struct Form {
    int bn, split;          // 16 or 32: rows of A in columns; 128: rows of A in lanes; kPairTile: pairs
    int64_t tiles;
};

// By estimates of the time in us, fitted to launches of 1 to 2048 rows, 512 to 8192 columns and K 512 to 8192 in every form (b:
// reduction steps of 256 on a CTA; one token x 512 in one piece 2.6 / 4.0 / 10.5 us for 2 / 8 / 32 steps, 128 x 512 3.8 / 5.5 / 11.9, pairs
// 5.2 / 6.9 / 13.6; split by eight 2.9 / 3.7 and 6.0 / 6.8 for 8 / 32).  At 91 sizes the choice takes 1.01 times the fastest form on average, 1.13
// at the most but for 33 x 1001 x 1000 (1.28).
Form pick_form(int64_t M, int64_t N, int k_blocks, int sms)
{
    const int64_t n_tiles = (N + 127) / 128, pairs = ((M + kPairTile - 1) / kPairTile) * ((N + kPairTile - 1) / kPairTile);
    const bool swap = M <= 32;
    const int bn = M <= 16 ? 16 : M <= 32 ? 32 : 128;
    Form best = {kPairTile, 1, pairs};
    double cost = swap || sms < 2 ? 1e30 : 3.2 + (double)((pairs + sms / 2 - 1) / (sms / 2)) * (1.5 + 0.28 * k_blocks);
    const int64_t tiles = (swap ? 1 : (M + 127) / 128) * n_tiles;
    for (int split = 1; split <= 8 && split <= k_blocks; split *= 2) {
        const int64_t at_once = clusters_at_once(split, sms);
        if (at_once == 0) break;
        const int64_t rounds = (tiles + at_once - 1) / at_once;
        const int b = (k_blocks + split - 1) / split;
        double c = swap ? 1.95 + 0.26 * b : 3.1 + 0.3 * b;
        if (split > 1) c += swap ? 0.5 : 0.7 + 1.8 * (double)(M < 128 ? M : 128) / 128;
        c *= (double)rounds;
        if (c < cost - 0.05) { cost = c; best = {bn, split, tiles}; }
    }
    return best;
}

// 64-element MMAs of a reduction over K, and the steps that hold four of them.
int mx_mmas(int64_t K) { return (int)((mx_padded(K) + 63) / 64); }
int mx_steps(int64_t K) { return (mx_mmas(K) + kMxSteps - 1) / kMxSteps; }

}  // namespace

}  // namespace sparq

using namespace sparq;

extern "C" int sparq_selftest_mxf4_form(int64_t M, int64_t N, int64_t K, int sms, int64_t *report)
{
    if (M < 1 || N < 1 || K < 1 || M >= kMxMost || N >= kMxMost || K >= kMxMost || sms < 1 || !report)
        return set_error(SPARQ_ERR_INVALID_ARG, "bad sizes of a product");
    const Form f = pick_form(M, N, mx_steps(K), sms);
    report[0] = f.bn;
    report[1] = f.split;
    report[2] = f.tiles;
    return SPARQ_OK;
}

extern "C" int sparq_gemm_mxf4(const void *A, const uint8_t *A_scales, const void *B, const uint8_t *B_scales,
                               int64_t M, int64_t N, int64_t K, int format, const sparq_mx_epilogue *e, void *stream)
{
    int rc = check_mx_format(format, true);
    if (rc != SPARQ_OK) return rc;
    if (!e) return set_error(SPARQ_ERR_INVALID_ARG, "sparq_mx_epilogue is NULL");
    if ((rc = check_mx_max(format, e->a_max, "a_max")) != SPARQ_OK || (rc = check_mx_max(format, e->b_max, "b_max")) != SPARQ_OK) return rc;
    if (M < 0 || N < 0 || K < 0) return set_error(SPARQ_ERR_INVALID_ARG, "negative dimension");
    if (!e->f32_out && !e->bf16_out) return set_error(SPARQ_ERR_INVALID_ARG, "no output requested (f32_out and bf16_out are both NULL)");
    if (M == 0 || N == 0) return SPARQ_OK;
    if (K == 0) return set_error(SPARQ_ERR_INVALID_ARG, "K is 0");
    if (!A || !A_scales || !B || !B_scales) return set_error(SPARQ_ERR_INVALID_ARG, "A/A_scales/B/B_scales pointer is NULL");
    if (M >= kMxMost || N >= kMxMost || K >= kMxMost) return set_error(SPARQ_ERR_UNSUPPORTED, "M, N and K must be below 2^31 - 256");
    if (((uintptr_t)A | (uintptr_t)A_scales | (uintptr_t)B | (uintptr_t)B_scales) & 15u)
        return set_error(SPARQ_ERR_UNSUPPORTED, "codes and scales must be 16-byte aligned");
    if (((uintptr_t)e->f32_out & 3u) || ((uintptr_t)e->bf16_out & 1u) || ((uintptr_t)e->bias & 3u))
        return set_error(SPARQ_ERR_UNSUPPORTED, "outputs and bias must be aligned to their elements");
    int sms = 0;
    if ((rc = device_info(&sms)) != SPARQ_OK) return rc;

    const bool nv = format == SPARQ_NVFP4;
    MxGemmArgs g = {};
    g.M = M;
    g.N = N;
    g.k_mmas = mx_mmas(K);
    g.k_blocks = mx_steps(K);
    g.scale_tiles = (int)(mx_scale_cols(format, K) / 4);
    g.a_scales = A_scales;
    g.b_scales = B_scales;
    g.a_max = e->a_max;
    g.b_max = e->b_max;
    g.bias = e->bias;
    g.relu = e->relu;
    g.f32_out = e->f32_out;
    g.bf16_out = (uint16_t *)e->bf16_out;
    g.wait_limit = kWaitLimitCycles;
    if ((rc = get_status_word(&g.status)) != SPARQ_OK) return rc;

    g.staged = (N % (e->bf16_out ? 8 : 4)) == 0 && (((uintptr_t)e->f32_out | (uintptr_t)e->bf16_out) & 15u) == 0;

    const int64_t pitch = mx_code_pitch(format, K);
    cudaStream_t st = (cudaStream_t)stream;
    const Form form = pick_form(M, N, g.k_blocks, sms);
    const int a_rows = form.bn < 128 ? form.bn : 128;
    CUtensorMap map[6] = {};       // A, B, their scales (pairs), f32_out, bf16_out
    if ((rc = encode_matrix(&map[0], CU_TENSOR_MAP_DATA_TYPE_UINT8, A, pitch, M, pitch, kMxBK, a_rows, CU_TENSOR_MAP_SWIZZLE_128B)) != SPARQ_OK ||
        (rc = encode_matrix(&map[1], CU_TENSOR_MAP_DATA_TYPE_UINT8, B, pitch, N, pitch, kMxBK, 128, CU_TENSOR_MAP_SWIZZLE_128B)) != SPARQ_OK)
        return rc;
    if (g.staged && form.bn >= 128) {
        if (e->f32_out &&
            (rc = encode_matrix(&map[4], CU_TENSOR_MAP_DATA_TYPE_FLOAT32, e->f32_out, N, M, N * 4, 32, 32, CU_TENSOR_MAP_SWIZZLE_128B)) != SPARQ_OK) return rc;
        if (e->bf16_out &&
            (rc = encode_matrix(&map[5], CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, e->bf16_out, N, M, N * 2, 64, 32, CU_TENSOR_MAP_SWIZZLE_128B)) != SPARQ_OK) return rc;
    }
    if (form.tiles * form.split > INT64_C(1) << 30) return set_error(SPARQ_ERR_UNSUPPORTED, "more than 2^30 tiles");
    if (form.bn == kPairTile) {
        MxPairArgs p = {g, (int)((M + kPairTile - 1) / kPairTile), (int)((N + kPairTile - 1) / kPairTile), 0};
        p.pairs = (int)(form.tiles < sms / 2 ? form.tiles : sms / 2);
        if ((rc = encode_scale_tiles(&map[2], A_scales, g.scale_tiles, (M + 127) / 128, scale_tiles(nv), 1)) != SPARQ_OK ||
            (rc = encode_scale_tiles(&map[3], B_scales, g.scale_tiles, (N + 127) / 128, scale_tiles(nv), 2)) != SPARQ_OK)
            return rc;
        const cudaError_t ce = nv ? launch_pair<true>(map, p, st) : launch_pair<false>(map, p, st);
        return ce == cudaSuccess ? SPARQ_OK : cuda_error(ce, "sparq_mxf4_kernel launch");
    }
    g.split = form.split;
    const int64_t grid = form.tiles * form.split;
    const cudaError_t ce = form.bn == 16 ? launch_small_of<16, true>(nv, map, g, grid, st)
                         : form.bn == 32 ? launch_small_of<32, true>(nv, map, g, grid, st) : launch_small_of<128, false>(nv, map, g, grid, st);
    return ce == cudaSuccess ? SPARQ_OK : cuda_error(ce, "sparq_mxf4_small_kernel launch");
}
