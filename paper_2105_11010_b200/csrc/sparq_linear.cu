// Host side of sparq_linear and sparq_linear_wgrad: validation, choice of form, launch.
#include <math.h>

#include "sparq_linear_small_kernel.cuh"
#include "sparq_linear_wgrad_kernel.cuh"

namespace sparq {

namespace {

int check_half(int dtype)
{
    if (dtype != SPARQ_DTYPE_BF16 && dtype != SPARQ_DTYPE_F16) return set_error(SPARQ_ERR_INVALID_ARG, "dtype %d is neither SPARQ_DTYPE_BF16 nor SPARQ_DTYPE_F16", dtype);
    return SPARQ_OK;
}

CUtensorMapDataType map_type(int dtype)
{
    return dtype == SPARQ_DTYPE_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : dtype == SPARQ_DTYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
}

// An operand that TMA reads: `rows` rows of `cols` elements; *ld becomes that of a single row where there is no other.
int check_operand(const char *name, const void *p, int64_t rows, int64_t cols, int64_t *ld)
{
    if (rows == 1) *ld = round_up64(cols, 8);
    if (*ld < cols) return set_error(SPARQ_ERR_INVALID_ARG, "the leading dimension of %s (%lld) is less than its columns (%lld)", name, (long long)*ld, (long long)cols);
    if (*ld % 8 || ((uintptr_t)p & 15u)) return set_error(SPARQ_ERR_UNSUPPORTED, "%s must be 16-byte aligned and its leading dimension a multiple of 8", name);
    if (*ld > INT64_C(1) << 38) return set_error(SPARQ_ERR_UNSUPPORTED, "the leading dimension of %s is %lld", name, (long long)*ld);
    return SPARQ_OK;
}

int check_output(const char *name, const void *p, int dtype, int64_t rows, int64_t cols, int64_t *ld)
{
    if (rows == 1) *ld = cols;
    if (*ld < cols) return set_error(SPARQ_ERR_INVALID_ARG, "the leading dimension of %s (%lld) is less than its columns (%lld)", name, (long long)*ld, (long long)cols);
    if ((uintptr_t)p & (uintptr_t)(dtype_width(dtype) - 1)) return set_error(SPARQ_ERR_UNSUPPORTED, "%s must be aligned to its elements", name);
    return check_mx_extent(rows, cols, *ld);
}

int check_groups(const int32_t *offsets, int64_t *groups)
{
    if (!offsets) *groups = 1;
    if (*groups < 1) return set_error(SPARQ_ERR_INVALID_ARG, "offsets of no experts");
    if (*groups > SPARQ_MAX_EXPERTS) return set_error(SPARQ_ERR_UNSUPPORTED, "%lld experts, %d at the most", (long long)*groups, SPARQ_MAX_EXPERTS);
    if ((uintptr_t)offsets & 3u) return set_error(SPARQ_ERR_UNSUPPORTED, "offsets must be 4-byte aligned");
    return SPARQ_OK;
}

// Tiles of `rows` rows that M rows of `groups` experts may make.
int64_t most_tiles(int64_t M, int64_t groups, int64_t rows) { return groups == 1 ? (M + rows - 1) / rows : (groups < M ? groups : M) + M / rows; }

template <class Kernel, class... Args>
cudaError_t launch_big(Kernel kernel, bool (&attr_set)[64], int grid, int cluster, int threads, int smem, cudaStream_t st, const Args &...args)
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64 || !attr_set[dev]) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64) attr_set[dev] = true;
    }
    return launch_overlapped_cluster(kernel, grid, cluster, threads, smem, st, args...);
}

// Parts that the steps of each expert's rows are cut into, where the tiles leave pairs idle: by estimates of the time in us.  Their sums take at most the
// scratch memory that the library keeps between synchronizations.
int pick_parts(int64_t M, int64_t tiles, int64_t elements, int64_t groups, int sms)
{
    const int64_t steps = (M / groups + kWgTokens - 1) / kWgTokens, pairs = sms / 2;
    int best = 1;
    double cost = 1e300;
    for (int parts = 1; parts <= 64 && parts * 4 <= steps + 3; ++parts) {
        if (parts > 1 && parts * elements * 4 > INT64_C(200) << 20) break;
        const double rounds = (double)((tiles * parts + pairs - 1) / pairs), b = (double)((steps + parts - 1) / parts);
        const double c = rounds * (2.5 + 0.33 * b) + (parts > 1 ? 3.0 + (double)(parts + 1) * (double)elements * 4.0 / 5.0e6 : 0.0);
        if (c < 0.97 * cost) { cost = c; best = parts; }
    }
    return best;
}

constexpr int kLinMaxDynSmem = 232448 - 2048;

struct LinForm {
    int bn, split;              // 16, 32, 64: tokens in columns; 128: tokens in lanes; kLinTile: pairs
    int64_t tiles;              // at the most, where experts' rows are cut on the device
    int per_sm;                 // CTAs that share an SM
};

// By estimates of the time in us, fitted to launches of 1 to 1024 rows, 512 to 8192 columns and K 1000 to 4096, and of 8 to 8192 rows of 16 and 64
// experts, in every form (b: reduction steps of 64 on a CTA; 16 x 1024, K 1024 in one piece 10.2 us, split by eight 5.0; 250 x 4096, K 4096 128-row
// tiles split by two 16.7, tokens in 64 columns 26; 512 rows of 64 experts, 1408 x 2048: 16 columns 63, 128 rows 80, pairs 88).  At 66 sizes the choice takes 1.03 times
// the fastest form on average, 1.28 at the most.  Experts' rows are taken to be spread evenly: the last tile of each is half full.
LinForm pick_linear(int64_t M, int64_t N, int k_blocks, int64_t groups, int sms)
{
    const int64_t n128 = (N + 127) / 128, n256 = (N + 255) / 256, touched = groups < M ? groups : M;
    const double each = (double)M / (double)touched;
    auto row_tiles = [&](int rows) { return groups == 1 ? (double)((M + rows - 1) / rows) : (double)touched * (each / rows + 0.5 > 1.0 ? each / rows + 0.5 : 1.0); };
    const double floor = 3.0 + (double)touched * (double)N * k_blocks * (2.0 * kLinBK / 5.6e6);       // the weights from HBM
    LinForm best = {};
    double cost = 1e300;
    auto consider = [&](double us, LinForm f) {
        const double c = (us > floor ? us : floor) + 0.1 * us;
        if (c < cost - 0.02) { cost = c; best = f; }
    };
    consider(3.6 + ceil(row_tiles(kLinTile) * (double)n256 / (sms / 2)) * (4.5 + 0.282 * k_blocks), {kLinTile, 1, most_tiles(M, groups, kLinTile) * n256, 1});
    for (int bn = 16; bn <= 128; bn *= 2) {
        if (bn < 128 && each > 8.0 * bn) continue;
        for (int split = 1; split <= (bn == 128 ? 4 : 8) && split <= k_blocks; split *= 2) {
            const int64_t tiles = most_tiles(M, groups, bn) * n128, at_once = clusters_at_once(split, sms);
            const int per_sm = bn < 128 && tiles > at_once ? 2 : 1, b = (k_blocks + split - 1) / split;
            if (at_once == 0 || (split > 1 && tiles > at_once * per_sm)) break;
            const double rounds = ceil(row_tiles(bn) * (double)n128 / (double)(at_once * per_sm)), cols = each < bn ? each : bn;
            if (bn == 128)
                consider(-1.3 + rounds * (6.3 + 0.256 * b + (split > 1 ? 0.5 + 2.1 * cols / 128 : 0.0)), {bn, split, tiles, per_sm});
            else
                consider(-0.4 + rounds * (1.5 + (per_sm == 1 ? 0.263 : 0.364) * b + (per_sm == 1 ? 0.13 : 0.195) * cols / split + 0.0014 * bn * b) +
                             (split > 1 ? 2.2 + 0.018 * cols : 0.0),
                         {bn, split, tiles, per_sm});
        }
    }
    return best;
}

template <int BN, bool SWAP, bool W_KN, bool F32, bool KEEP>
cudaError_t launch_lin_small(const LinForm &f, const LinArgs &g, cudaStream_t st, const CUtensorMap &map_x, const CUtensorMap &map_w, const CUtensorMap &map_out)
{
    static bool attr_set[64] = {};
    const int64_t C = SWAP ? g.M : g.N;
    const int recv = lin_recv_bytes(lin_own_groups((int)(C < BN ? C : BN), f.split, SWAP), f.split, SWAP), stage = lin_small_stage(BN);
    // (each CTA's barriers and 1 KB that the system takes are beside its dynamic memory)
    const int room = (f.per_sm == 2 ? 112 * 1024 : kLinMaxDynSmem) - 1024 - recv, steps = (g.k_blocks + f.split - 1) / f.split;
    LinSmallArgs p = {g, room / stage, f.split};
    if (p.stages > steps) p.stages = steps;
    if (p.stages > kMaxStages) p.stages = kMaxStages;
    const int smem = 1024 + p.stages * stage + recv;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    auto kernel = sparq_linear_small_kernel<BN, SWAP, W_KN, F32, KEEP>;
    if (dev < 0 || dev >= 64 || !attr_set[dev]) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kLinMaxDynSmem);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64) attr_set[dev] = true;
    }
    return launch_overlapped_cluster(kernel, (int)(f.tiles * f.split), f.split, lin_small_threads(SWAP), smem, st, map_x, map_w, map_out, p);
}

template <bool W_KN, bool F32, bool KEEP, bool PIECES>
cudaError_t launch_pairs(const LinArgs &g, cudaStream_t st, const CUtensorMap &map_x, const CUtensorMap &map_w, const CUtensorMap &map_out)
{
    static bool attr_set[64] = {};
    return launch_big(sparq_linear_kernel<W_KN, F32, KEEP, PIECES>, attr_set, 2 * g.units, 2, lin_threads(PIECES), kLinSmem, st, map_x, map_w, map_out, g);
}

template <bool W_KN, bool F32, bool KEEP>
cudaError_t launch_linear(const LinForm &f, const LinArgs &g, cudaStream_t st, const CUtensorMap &map_x, const CUtensorMap &map_w, const CUtensorMap &map_out)
{
    switch (f.bn) {
    case 16: return launch_lin_small<16, true, W_KN, F32, KEEP>(f, g, st, map_x, map_w, map_out);
    case 32: return launch_lin_small<32, true, W_KN, F32, KEEP>(f, g, st, map_x, map_w, map_out);
    case 64: return launch_lin_small<64, true, W_KN, F32, KEEP>(f, g, st, map_x, map_w, map_out);
    case 128: return launch_lin_small<128, false, W_KN, F32, KEEP>(f, g, st, map_x, map_w, map_out);
    default: return g.k_blocks > g.piece ? launch_pairs<W_KN, F32, KEEP, true>(g, st, map_x, map_w, map_out) : launch_pairs<W_KN, F32, KEEP, false>(g, st, map_x, map_w, map_out);
    }
}
template <bool W_KN>
cudaError_t launch_linear_of(bool f32, bool keep, const LinForm &f, const LinArgs &g, cudaStream_t st, const CUtensorMap &map_x, const CUtensorMap &map_w,
                             const CUtensorMap &map_out)
{
    if (f32) return keep ? launch_linear<W_KN, true, true>(f, g, st, map_x, map_w, map_out) : launch_linear<W_KN, true, false>(f, g, st, map_x, map_w, map_out);
    return keep ? launch_linear<W_KN, false, true>(f, g, st, map_x, map_w, map_out) : launch_linear<W_KN, false, false>(f, g, st, map_x, map_w, map_out);
}

}  // namespace

}  // namespace sparq

using namespace sparq;

extern "C" int sparq_selftest_linear_form(int64_t M, int64_t N, int64_t K, int64_t groups, int sms, int64_t *report)
{
    if (M < 1 || N < 1 || K < 1 || M >= kMxMost || N >= kMxMost || K >= kMxMost || groups < 1 || groups > SPARQ_MAX_EXPERTS || sms < 2 || !report)
        return set_error(SPARQ_ERR_INVALID_ARG, "bad sizes of a product");
    const LinForm f = pick_linear(M, N, (int)((K + kLinBK - 1) / kLinBK), groups, sms);
    report[0] = f.bn;
    report[1] = f.split;
    report[2] = f.tiles;
    report[3] = f.per_sm;
    return SPARQ_OK;
}

extern "C" int sparq_linear(const void *x, int64_t ldx, const void *w, int64_t ldw, int64_t w_stride, int transposed, int dtype, int64_t M, int64_t N, int64_t K,
                            const int32_t *offsets, int64_t groups, const sparq_linear_epilogue *e, void *stream)
{
    int rc = check_half(dtype);
    if (rc != SPARQ_OK) return rc;
    if (!e) return set_error(SPARQ_ERR_INVALID_ARG, "sparq_linear_epilogue is NULL");
    if (M < 0 || N < 0 || K < 0) return set_error(SPARQ_ERR_INVALID_ARG, "negative dimension");
    if (e->act < SPARQ_ACT_IDENTITY || e->act > SPARQ_ACT_GELU) return set_error(SPARQ_ERR_INVALID_ARG, "act %d is not one of SPARQ_ACT_*", e->act);
    if (e->out_dtype != dtype && e->out_dtype != SPARQ_DTYPE_F32) return set_error(SPARQ_ERR_INVALID_ARG, "out_dtype %d is neither the operands' type nor SPARQ_DTYPE_F32", e->out_dtype);
    if (!e->z_codes != !e->z_scales) return set_error(SPARQ_ERR_INVALID_ARG, "z_codes and z_scales come together");
    if ((rc = check_groups(offsets, &groups)) != SPARQ_OK) return rc;
    if (M == 0 || N == 0) return SPARQ_OK;
    if (K == 0) return set_error(SPARQ_ERR_INVALID_ARG, "K is 0");
    if (!x || !w || !e->out) return set_error(SPARQ_ERR_INVALID_ARG, "x/w/out pointer is NULL");
    if (M >= kMxMost || N >= kMxMost || K >= kMxMost) return set_error(SPARQ_ERR_UNSUPPORTED, "M, N and K must be below 2^31 - 256");
    const int64_t w_rows = transposed ? K : N, w_cols = transposed ? N : K;
    int64_t ldo = e->ldo, ldr = e->ldr;
    if ((rc = check_operand("x", x, M, K, &ldx)) != SPARQ_OK || (rc = check_operand("w", w, w_rows, w_cols, &ldw)) != SPARQ_OK ||
        (rc = check_output("out", e->out, e->out_dtype, M, N, &ldo)) != SPARQ_OK ||
        (e->residual && (rc = check_output("residual", e->residual, e->out_dtype, M, N, &ldr)) != SPARQ_OK))
        return rc;
    if (groups == 1) w_stride = w_rows * ldw;
    if (w_stride < (w_rows - 1) * ldw + w_cols) return set_error(SPARQ_ERR_INVALID_ARG, "w_stride (%lld) is less than a weight matrix", (long long)w_stride);
    if (w_stride % 8 || w_stride > INT64_C(1) << 38) return set_error(SPARQ_ERR_UNSUPPORTED, "w_stride must be a multiple of 8 and at most 2^38");
    if (e->out == x || e->out == w) return set_error(SPARQ_ERR_INVALID_ARG, "out is x or w");
    if (e->residual == e->out && ldr != ldo) return set_error(SPARQ_ERR_INVALID_ARG, "out in place of residual has its leading dimension");
    if ((uintptr_t)e->bias & 3u) return set_error(SPARQ_ERR_UNSUPPORTED, "bias must be 4-byte aligned");
    if (((uintptr_t)e->z_codes | (uintptr_t)e->z_scales) & 15u) return set_error(SPARQ_ERR_UNSUPPORTED, "z_codes and z_scales must be 16-byte aligned");
    if (e->z_codes && (rc = check_mx_extent(M, N, mx_padded(N))) != SPARQ_OK) return rc;
    int sms = 0;
    if ((rc = device_info(&sms)) != SPARQ_OK) return rc;
    if (sms < 2) return set_error(SPARQ_ERR_UNSUPPORTED, "a device of one multiprocessor");

    LinArgs g = {};
    g.M = M;
    g.N = N;
    g.k_mmas = (int)((K + 15) / 16);
    g.k_blocks = (int)((K + kLinBK - 1) / kLinBK);
    g.piece = lin_piece(K, e->out_dtype == SPARQ_DTYPE_F32 || e->z_codes);
    g.offsets = offsets;
    g.groups = (int)groups;
    g.bf16 = dtype == SPARQ_DTYPE_BF16;
    g.bias = e->bias;
    g.act = e->act;
    g.residual = e->residual;
    g.ldr = ldr;
    g.out = e->out;
    g.ldo = ldo;
    g.z_codes = e->z_codes;
    g.z_scales = e->z_scales;
    g.z_pitch = mx_code_pitch(SPARQ_MXINT8, N);
    g.z_spitch = mx_scale_cols(SPARQ_MXINT8, N);
    const int width = dtype_width(e->out_dtype);
    g.staged = (((uintptr_t)e->out | (uintptr_t)(ldo * width)) & 15u) == 0;
    g.wait_limit = kWaitLimitCycles;
    if ((rc = get_status_word(&g.status)) != SPARQ_OK) return rc;

    cudaStream_t st = (cudaStream_t)stream;
    const LinForm form = pick_linear(M, N, g.k_blocks, groups, sms);
    if (form.tiles * form.split > INT64_C(1) << 30) return set_error(SPARQ_ERR_UNSUPPORTED, "more than 2^30 tiles");
    const int box_cols = form.bn == kLinTile ? kLinTile : 128, x_rows = form.bn < 128 ? form.bn : 128;
    g.n_tiles = (int)((N + box_cols - 1) / box_cols);
    g.units = (int)(form.tiles < sms / 2 ? form.tiles : sms / 2);
    CUtensorMap map_x = {}, map_w = {}, map_out = {};
    if ((rc = encode_matrix(&map_x, map_type(dtype), x, K, M, ldx * 2, kLinBK, x_rows, CU_TENSOR_MAP_SWIZZLE_128B)) != SPARQ_OK ||
        (rc = encode_matrices(&map_w, map_type(dtype), w, w_cols, w_rows, groups, ldw * 2, w_stride * 2, 64, transposed ? kLinBK : 128, CU_TENSOR_MAP_SWIZZLE_128B)) != SPARQ_OK)
        return rc;
    if (g.staged && form.bn >= 128 &&
        (rc = encode_matrix(&map_out, map_type(e->out_dtype), e->out, N, M, ldo * width, 128 / width, 32, CU_TENSOR_MAP_SWIZZLE_128B)) != SPARQ_OK)
        return rc;
    const bool f32 = e->out_dtype == SPARQ_DTYPE_F32, keep = e->z_codes != nullptr;
    const cudaError_t ce = transposed ? launch_linear_of<true>(f32, keep, form, g, st, map_x, map_w, map_out) : launch_linear_of<false>(f32, keep, form, g, st, map_x, map_w, map_out);
    return ce == cudaSuccess ? SPARQ_OK : cuda_error(ce, "linear layer's kernel launch");
}

extern "C" int sparq_linear_wgrad(const void *dy, int64_t lddy, const void *x, int64_t ldx, int dtype, int64_t M, int64_t N, int64_t K, const int32_t *offsets, int64_t groups,
                                  int accumulate, float *dw, float *dbias, void *stream)
{
    int rc = check_half(dtype);
    if (rc != SPARQ_OK) return rc;
    if (M < 0 || N < 0 || K < 0) return set_error(SPARQ_ERR_INVALID_ARG, "negative dimension");
    if ((rc = check_groups(offsets, &groups)) != SPARQ_OK) return rc;
    if (N == 0 || (K == 0 && !dbias)) return SPARQ_OK;
    if (K > 0 && !dw) return set_error(SPARQ_ERR_INVALID_ARG, "dw is NULL");
    if (((uintptr_t)dw | (uintptr_t)dbias) & 3u) return set_error(SPARQ_ERR_UNSUPPORTED, "dw and dbias must be 4-byte aligned");
    if (M >= kMxMost || N >= kMxMost || K >= kMxMost) return set_error(SPARQ_ERR_UNSUPPORTED, "M, N and K must be below 2^31 - 256");
    if ((__int128)groups * N * (K + 1) > INT64_C(1) << 58) return set_error(SPARQ_ERR_UNSUPPORTED, "gradients of more elements than any device holds");
    cudaStream_t st = (cudaStream_t)stream;
    if (M == 0) {           // sums over no rows
        if (accumulate) return SPARQ_OK;
        cudaError_t e = K > 0 ? cudaMemsetAsync(dw, 0, (size_t)groups * (size_t)N * (size_t)K * sizeof(float), st) : cudaSuccess;
        if (e == cudaSuccess && dbias) e = cudaMemsetAsync(dbias, 0, (size_t)groups * (size_t)N * sizeof(float), st);
        return e == cudaSuccess ? SPARQ_OK : cuda_error(e, "cudaMemsetAsync(dw, dbias)");
    }
    if (!dy || (K > 0 && !x)) return set_error(SPARQ_ERR_INVALID_ARG, "dy/x pointer is NULL");
    if ((rc = check_operand("dy", dy, M, N, &lddy)) != SPARQ_OK || (K > 0 && (rc = check_operand("x", x, M, K, &ldx)) != SPARQ_OK)) return rc;
    int sms = 0;
    if ((rc = device_info(&sms)) != SPARQ_OK) return rc;
    if (sms < 2) return set_error(SPARQ_ERR_UNSUPPORTED, "a device of one multiprocessor");

    if (K > 0) {
        LinWgradArgs g = {};
        g.M = M;
        g.N = N;
        g.K = K;
        g.offsets = offsets;
        g.groups = (int)groups;
        g.bf16 = dtype == SPARQ_DTYPE_BF16;
        g.accumulate = accumulate != 0;
        g.dw = dw;
        g.n_tiles = (int)((N + kWgTile - 1) / kWgTile);
        g.k_tiles = (int)((K + kWgTile - 1) / kWgTile);
        const int64_t tiles = (int64_t)g.n_tiles * g.k_tiles * groups, elements = groups * N * K;
        g.wait_limit = kWaitLimitCycles;
        if ((rc = get_status_word(&g.status)) != SPARQ_OK) return rc;
        g.parts = pick_parts(M, tiles, elements, groups, sms);
        if (tiles * g.parts > INT64_C(1) << 29) return set_error(SPARQ_ERR_UNSUPPORTED, "more than 2^29 tiles");
        LwMaps maps = {};
        CUtensorMap map_dw = {};
        const int rows[kLwBoxes] = {kWgTokens, 16, 8, 4, 2, 1};
        for (int b = 0; b < (offsets ? kLwBoxes : 1); ++b)
            if ((rc = encode_matrix(&maps.dy[b], map_type(dtype), dy, N, M, lddy * 2, 64, rows[b], CU_TENSOR_MAP_SWIZZLE_128B)) != SPARQ_OK ||
                (rc = encode_matrix(&maps.x[b], map_type(dtype), x, K, M, ldx * 2, 64, rows[b], CU_TENSOR_MAP_SWIZZLE_128B)) != SPARQ_OK)
                return rc;
        for (int b = 1; b < kLwBoxes && !offsets; ++b) {     // not used
            maps.dy[b] = maps.dy[0];
            maps.x[b] = maps.x[0];
        }
        // Memory for the parts' sums is scratch.  Without any (a stream that is being captured) the parts add to dw one launch after the other: the
        // same sums in the same order.
        float *const sums = g.parts > 1 ? (float *)workspace_alloc((size_t)g.parts * (size_t)elements * sizeof(float), st) : nullptr;
        const int launches = sums ? 1 : g.parts;
        g.count = sums ? g.parts : 1;
        g.part_stride = elements;
        rc = SPARQ_OK;
        for (int l = 0; l < launches && rc == SPARQ_OK; ++l) {
            g.part = l;
            g.dw = sums ? sums : dw;
            g.accumulate = sums ? 0 : accumulate != 0 || l > 0;
            g.staged = !g.accumulate && K % 4 == 0 && ((uintptr_t)g.dw & 15u) == 0;
            if (g.staged && (rc = encode_matrices(&map_dw, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, g.dw, K, N, groups * g.count, K * 4, N * K * 4, 32, 32, CU_TENSOR_MAP_SWIZZLE_128B)) != SPARQ_OK)
                break;
            // Where a last round would leave half of the pairs idle its tiles come in halves, 256 x 128 (16384 x 4096 x 4096, 256 tiles on 74 pairs:
            // 395 us, whole 426).
            const int64_t items = tiles * g.count, pairs = sms / 2, rest = items % pairs;
            g.whole = (int)(2 * rest <= pairs ? items - rest : items);
            g.pairs = (int)(2 * items - g.whole < pairs ? 2 * items - g.whole : pairs);
            static bool attr_set[64] = {};
            const cudaError_t e = launch_big(sparq_linear_wgrad_kernel, attr_set, 2 * g.pairs, 2, kLwThreads, kLwSmem, st, maps, map_dw, g);
            if (e != cudaSuccess) rc = cuda_error(e, "sparq_linear_wgrad_kernel launch");
        }
        if (sums && rc == SPARQ_OK) {
            const int64_t blocks = (elements / 4 + 256) / 256;
            const cudaError_t e = launch_overlapped(linear_add_parts_kernel, (int)(blocks < 8 * sms ? blocks : 8 * sms), 256, 0, st, (const float *)sums, elements, g.parts,
                                                    (int)(accumulate != 0), dw);
            if (e != cudaSuccess) rc = cuda_error(e, "linear_add_parts_kernel launch");
        }
        workspace_free(sums, st);
        if (rc != SPARQ_OK) return rc;
    }
    if (dbias) {
        BiasGrad b = {dy, M, N, lddy, offsets, (int)groups, (int)((N + kBiasCols - 1) / kBiasCols), 1, accumulate != 0, dbias};
        // enough CTAs to keep HBM busy, each with a few hundred rows at least
        while (b.split < 8 && clusters_at_once(2 * b.split, sms) > 0 && (int64_t)b.col_tiles * groups * b.split < 8 * sms && M / groups >= 256 * b.split) b.split *= 2;
        const int64_t grid = (int64_t)b.col_tiles * groups * b.split;
        if (grid > INT64_C(1) << 30) return set_error(SPARQ_ERR_UNSUPPORTED, "more than 2^30 tiles");
        const cudaError_t e = launch_overlapped_cluster(dtype == SPARQ_DTYPE_BF16 ? linear_bias_grad_kernel<true> : linear_bias_grad_kernel<false>, (int)grid, b.split,
                                                        kBiasThreads, 0, st, b);
        if (e != cudaSuccess) return cuda_error(e, "linear_bias_grad_kernel launch");
    }
    return SPARQ_OK;
}
