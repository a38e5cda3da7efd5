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

struct WgradForm {
    bool pairs, expand;     // pairs of CTAs on 256 x 256 tiles, X expanded to bf16 first
    int split, parts;
    int64_t tiles, whole;   // whole: tiles in front that are not cut into the parts
};

// X in bf16, and the sums of the parts: one piece of memory.
struct Scratch {
    size_t x, sums;
    size_t bytes() const { return x + sums; }
};
Scratch scratch_of(const WgradForm &f, int64_t M, int64_t N, int64_t K)
{
    auto round = [](size_t b) { return (b + 255) / 256 * 256; };
    return {f.expand ? round((size_t)M * (size_t)mx_padded(K) * 2) : 0,
            f.parts == 1 ? 0
            : f.whole ? (size_t)(f.parts - 1) * (size_t)(f.tiles - f.whole) * kWgTile * kWgTile * sizeof(float)
                      : round((size_t)f.parts * (size_t)N * (size_t)K * sizeof(float))};
}

// By estimates of the time in us, fitted to launches of 64 to 100352 tokens and 64 x 256 to 2048 x 2048 outputs in every form.  At 33 sizes of
// 64 to 131072 tokens and 64 x 64 to 4096 x 4096 outputs the choice takes 1.03 times the fastest form on average, 1.11 at the most but for 80000 x
// 64 x 64 (1.37: 128 parts for 12 in clusters of eight).  A step of 64 tokens takes a tile 0.45 us (128 x 128, transformed on the way),
// 0.53 (256 x 256) and 0.36 (256 x 256, expanded first).  16384 x 1024 x 1024: pairs in one part 139 us, in four 47, expanded first 89 and 42;
// 4096 x 128 x 1152: 128 x 128 30 us, in eight parts 10.7, split in clusters of eight 11.3.  A form whose scratch memory the library does not
// give (kWorkspaceMaxBytes) is none: it would run as another, without it.
WgradForm pick_wgrad(int64_t M, int64_t N, int64_t K, int blocks, int sms)
{
    WgradForm best = {};
    double cost = 1e30;
    const bool x16_fits = (double)M * (double)mx_padded(K) * 2.0 <= (double)kWorkspaceMaxBytes;
    auto consider = [&](double c, const WgradForm &f) {
        if (c < cost - 0.05 && (!f.expand || x16_fits) && scratch_of(f, M, N, K).bytes() <= kWorkspaceMaxBytes) { cost = c; best = f; }
    };
    const int64_t small = (N + 127) / 128 * ((K + 127) / 128), large = (N + 255) / 256 * ((K + 255) / 256), pairs = sms / 2;
    const double expand = 1.5 + (double)M * (double)K * 3.0 / 6.0e6;
    for (int parts = 1; parts <= 128 && parts * 8 <= blocks + 7; parts += parts < 8 ? 1 : parts < 32 ? 4 : 16) {
        if (parts > 1 && (double)parts * (double)N * (double)K * 4.0 > (double)kWorkspaceMaxBytes) break;
        const int b = (blocks + parts - 1) / parts;
        const double join = parts > 1 ? 2.5 + (double)(parts + 1) * (double)N * (double)K * 4.0 / 5.0e6 : 0.0;
        // (the shorter parts have blocks / parts steps, and every CTA of a cluster needs one)
        for (int split = 1; split <= 8 && split <= blocks / parts; split *= 2) {
            const int64_t at_once = clusters_at_once(split, sms);
            if (at_once == 0) break;
            const int64_t rounds = (small * parts + at_once - 1) / at_once;
            const double c = join + 1.0 + (double)rounds * (4.6 + 0.45 * ((b + split - 1) / split) + (split > 1 ? 1.5 : 0.0));
            consider(c, {false, false, split, parts, small, 0});
        }
        if (pairs == 0) continue;
        const int64_t rounds = (large * parts + pairs - 1) / pairs;
        consider(join + 7.0 + (double)rounds * 0.53 * b, {true, false, 1, parts, large, 0});
        consider(join + 7.0 + expand + (double)rounds * 0.36 * b, {true, true, 1, parts, large, 0});
    }
    // Whole tiles but for a last round that leaves most pairs without one, whose tiles are cut (256 tiles on 74 pairs: 3 rounds and
    // a half for 4; 16384 x 4096 x 4096 396 us, uncut 417, in two parts throughout 435; 4100 x 2560 x 2040 58 and, uncut, 70).
    const int64_t tail = pairs ? large % pairs : 0;
    for (int parts = 2; parts <= 8 && parts * 8 <= blocks && large > pairs && tail > 0; ++parts) {
        const double b = (double)(large / pairs) * blocks + (double)((tail * parts + pairs - 1) / pairs) * ((blocks + parts - 1) / parts);
        const double join = 3.0 + (double)(2 * parts * tail) * (kWgTile * kWgTile * 4.0 / 5.0e6);
        consider(join + 7.0 + 0.53 * b, {true, false, 1, parts, large, large - tail});
        consider(join + 7.0 + expand + 0.36 * b, {true, true, 1, parts, large, large - tail});
    }
    return best;
}

}  // namespace

}  // namespace sparq

using namespace sparq;

extern "C" int64_t sparq_wgrad_mx8_workspace_bytes(int64_t M, int64_t N, int64_t K)
{
    if (M < 0 || N < 0 || K < 0) return set_error(SPARQ_ERR_INVALID_ARG, "negative dimension");
    if (M >= kMxMost || N >= kMxMost || K >= kMxMost) return set_error(SPARQ_ERR_UNSUPPORTED, "M, N and K must be below 2^31 - 256");
    if (M == 0 || N == 0 || K == 0) return 0;
    int sms = 0;
    const int rc = device_info(&sms);
    if (rc != SPARQ_OK) return rc;
    return (int64_t)scratch_of(pick_wgrad(M, N, K, (int)((M + kWgTokens - 1) / kWgTokens), sms), M, N, K).bytes();
}

extern "C" int sparq_selftest_wgrad_form(int64_t M, int64_t N, int64_t K, int sms, int64_t *report)
{
    if (M < 1 || N < 1 || K < 1 || M >= kMxMost || N >= kMxMost || K >= kMxMost || sms < 1 || !report)
        return set_error(SPARQ_ERR_INVALID_ARG, "bad sizes of a weight gradient");
    const WgradForm f = pick_wgrad(M, N, K, (int)((M + kWgTokens - 1) / kWgTokens), sms);
    const int64_t words[6] = {f.pairs ? f.expand ? 2 : 1 : 0, f.split, f.parts, f.tiles, f.whole, (int64_t)scratch_of(f, M, N, K).bytes()};
    for (int i = 0; i < 6; ++i) report[i] = words[i];
    return SPARQ_OK;
}

extern "C" int sparq_wgrad_mx8(const void *dy, int64_t lddy, const int8_t *codes, const uint8_t *scales,
                               int64_t M, int64_t N, int64_t K, int accumulate, float *dw, void *workspace, size_t workspace_bytes, void *stream)
{
    if (M < 0 || N < 0 || K < 0) return set_error(SPARQ_ERR_INVALID_ARG, "negative dimension");
    if (N == 0 || K == 0) return SPARQ_OK;
    if (!dw) return set_error(SPARQ_ERR_INVALID_ARG, "dw is NULL");
    if ((uintptr_t)dw & 3u) return set_error(SPARQ_ERR_UNSUPPORTED, "dw must be 4-byte aligned");
    if (M >= kMxMost || N >= kMxMost || K >= kMxMost) return set_error(SPARQ_ERR_UNSUPPORTED, "M, N and K must be below 2^31 - 256");
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
    if ((rc = encode_matrix(&map_codes, CU_TENSOR_MAP_DATA_TYPE_UINT8, codes, pitch, M, pitch, kWgBN, kWgTokens, CU_TENSOR_MAP_SWIZZLE_128B)) != SPARQ_OK) return rc;
    if ((rc = encode_matrix(&map_scales, CU_TENSOR_MAP_DATA_TYPE_UINT8, scales, spitch, M, spitch, 16, kWgTokens, CU_TENSOR_MAP_SWIZZLE_NONE)) != SPARQ_OK) return rc;
    const WgradForm form = pick_wgrad(M, N, K, g.blocks, sms);
    const Scratch need = scratch_of(form, M, N, K);
    if (workspace && ((uintptr_t)workspace & 255u)) return set_error(SPARQ_ERR_UNSUPPORTED, "workspace must be 256-byte aligned");
    if (workspace && workspace_bytes < need.bytes())
        return set_error(SPARQ_ERR_INVALID_ARG, "workspace of %zu bytes, %zu are needed", workspace_bytes, need.bytes());
    g.parts = form.parts;
    g.split = form.split;
    if (form.tiles * form.parts * form.split > INT64_C(1) << 30) return set_error(SPARQ_ERR_UNSUPPORTED, "more than 2^30 tiles");
    // Memory for X in bf16 and for the parts' sums: the caller's, else scratch.  Without any (a stream that is being captured) X is expanded
    // stage by stage and the parts add to dw one launch after the other: the same sums in the same order.
    CUtensorMap map_x;
    const size_t bytes = need.bytes();
    void *const own = !workspace && bytes ? workspace_alloc(bytes, st) : nullptr;
    uint8_t *const room = (uint8_t *)(workspace ? workspace : own);
    void *const x = room && need.x ? room : nullptr;
    float *const sums = room && need.sums ? (float *)(room + need.x) : nullptr;
    rc = SPARQ_OK;
    if (x) {
        rc = sparq_dequantize_mx(codes, scales, M, K, SPARQ_MXINT8, nullptr, x, SPARQ_DTYPE_BF16, pitch, stream);
        if (rc == SPARQ_OK) rc = encode_matrix(&map_x, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, x, K, M, pitch * 2, 64, kWgTokens, CU_TENSOR_MAP_SWIZZLE_128B);
    }
    const int launches = sums ? 1 : g.parts;
    if (sums && form.whole == 0) {
        g.dw = sums;
        g.part_stride = N * K;
        g.accumulate = 0;
    }
    g.count = sums ? g.parts : 1;
    WgradPairArgs p = {g, (int)((N + kWgTile - 1) / kWgTile), (int)((K + kWgTile - 1) / kWgTile), 0, (int)form.whole, 0, form.whole ? sums : nullptr};
    for (int l = 0; l < launches && rc == SPARQ_OK; ++l) {
        g.part = l;
        if (!sums) g.accumulate = accumulate != 0 || l > 0;
        cudaError_t e;
        if (form.pairs) {
            p.g = g;
            p.skip = form.whole && l > 0;
            const int64_t items = (p.skip ? 0 : form.whole) + (form.tiles - form.whole) * g.count;
            p.pairs = (int)(items < sms / 2 ? items : sms / 2);
            static bool set_x[64] = {}, set_q[64] = {};
            e = x ? launch_wgrad(sparq_wgrad_kernel<true>, set_x, 2 * p.pairs, 2, kWgPairThreads, wgrad_smem(true), st, map_dy, map_x, map_x, p)
                  : launch_wgrad(sparq_wgrad_kernel<false>, set_q, 2 * p.pairs, 2, kWgPairThreads, wgrad_smem(false), st, map_dy, map_codes, map_scales, p);
        } else {
            static bool set[64] = {};
            e = launch_wgrad(sparq_wgrad_small_kernel, set, (int)(form.tiles * g.count * g.split), g.split, kWgThreads, 1024 + WgradSmall::kRings, st,
                             map_dy, map_codes, map_scales, g);
        }
        if (e != cudaSuccess) rc = cuda_error(e, "weight gradient kernel launch");
    }
    if (sums && form.whole && rc == SPARQ_OK) {
        const cudaError_t e = launch_overlapped(wgrad_add_tail_kernel, (int)(form.tiles - form.whole) * (kWgTile / kWgAddRows), kWgTile, 0, st, p);
        if (e != cudaSuccess) rc = cuda_error(e, "wgrad_add_tail_kernel launch");
    } else if (sums && rc == SPARQ_OK) {
        const int64_t threads = (N * K + 3) / 4, blocks = (threads + 255) / 256;
        const cudaError_t e = launch_overlapped(wgrad_add_parts_kernel, (int)(blocks < 8 * sms ? blocks : 8 * sms), 256, 0, st, (const float *)sums, N * K,
                                                g.parts, (int)(accumulate != 0), dw);
        if (e != cudaSuccess) rc = cuda_error(e, "wgrad_add_parts_kernel launch");
    }
    workspace_free(own, st);
    return rc;
}
