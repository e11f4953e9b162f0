// C ABI of the fptq library: argument validation, shape dispatch, error text.
// Every entry point validates first and launches afterwards, so a failing call writes nothing.
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <mutex>

#include "fptq_attention.h"
#include "fptq_common.h"
#include "fptq_testing.h"

namespace fptq {

static thread_local char g_err[256] = "";

void set_error(const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof g_err, fmt, ap);
    va_end(ap);
}

static int hip_fail(const char *what, hipError_t e)
{
    set_error("%s: %s", what, hipGetErrorString(e));
    return FPTQ_ERR_HIP;
}

static const int64_t MAX_ELEMS = (int64_t)1 << 40;
// INT32 accumulation is exact while 64 K < 2^31 (|q w| <= 64); with a zero point the epilogue forms
// acc - z * sum_k w, at most 128 K in magnitude.
static const int64_t MAX_K = ((int64_t)1 << 25) - 1, MAX_K_ZERO_POINT = ((int64_t)1 << 24) - 1;

// ---- per-device state.  Filled once per device under a lock; readers take the lock-free path afterwards.
static DeviceInfo g_devices[MAX_DEVICES];
static std::atomic<bool> g_device_ready[MAX_DEVICES];
static std::mutex g_device_mutex;

hipError_t device_info(const DeviceInfo **out)
{
    int dev = -1;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (dev < 0 || dev >= MAX_DEVICES) return hipErrorInvalidDevice;
    if (!g_device_ready[dev].load(std::memory_order_acquire)) {
        std::lock_guard<std::mutex> lock(g_device_mutex);
        if (!g_device_ready[dev].load(std::memory_order_relaxed)) {
            DeviceInfo info = {};
            info.device = dev;
            int cus = 0;
            if ((e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev)) != hipSuccess) return e;
            info.cus = cus > 0 ? cus : DEFAULT_CUS;
            if ((e = gemm_device_init(&info)) != hipSuccess) return e;
            if ((e = prefill_device_init()) != hipSuccess) return e;
            g_devices[dev] = info;
            g_device_ready[dev].store(true, std::memory_order_release);
        }
    }
    *out = &g_devices[dev];
    return hipSuccess;
}

int device_cus_or_default()
{
    const DeviceInfo *info;
    if (device_info(&info) != hipSuccess) {
        (void)hipGetLastError();     // a host-only query without a device must not leave a sticky error behind
        return DEFAULT_CUS;
    }
    return info->cus;
}

static int check_dims(const char *fn, int64_t a, int64_t b, const char *an, const char *bn)
{
    if (a < 1 || b < 1 || a > MAX_ELEMS / b) {
        set_error("%s: bad shape %s=%lld %s=%lld", fn, an, (long long)a, bn, (long long)b);
        return FPTQ_ERR_SHAPE;
    }
    return FPTQ_OK;
}

static int check_align(const char *fn, const void *p, unsigned a, const char *name)
{
    if (reinterpret_cast<uintptr_t>(p) & (a - 1)) {
        set_error("%s: %s must be %u-byte aligned", fn, name, a);
        return FPTQ_ERR_ALIGN;
    }
    return FPTQ_OK;
}

// The few-token kernel serves up to 32 tokens and, where its workgroups of 32 channels are a single round of the CUs, up to 64;
// above that, or whenever a prefill tile shape is forced, the MFMA GEMM runs: its 64 x 64 and 128 x 64 tiles with four K groups
// are faster from 65 tokens on everywhere, and from 33 tokens on where a second round begins (33 to 64 tokens over cold weights, few tokens /
// tiles: 8168 channels of K = 3872 7.4 us / 8.8, 9784 x 4968 13.1 / 10.4, 8384 x 8416 18.5 / 13.5, 8824 x 14944 31.1 / 20.2; of 81 matrices of 8200 to
// 10239 channels the tiles take 12 to 36 % less on each).  They are also faster with 17 to 32 tokens against more than 12288 channels of fewer than
// 16 K tiles, too few for the 16 waves that share a K otherwise: 15208 x 992 6.2 us / 5.7, 29040 x 1352 11.7 / 8.5, 36536 x 1384 14.0 / 13.0, 57288 x 736
// 17.3 / 11.5; 2 % more to 34 % less on 87 matrices of up to 62000 channels, and up to 6 % more below 12288: where both kernels
// fill the 256 CUs that it was measured on.  With fewer of them (a partitioned card) nothing was measured, and the line stays.
static bool few_token_shape(int64_t M, int64_t N, int64_t K)
{
    if (M > 64 || N > (1 << 24)) return M <= 32;
    if (M > 32) return N <= 32 * (int64_t)device_cus_or_default() || (K > 65535 && N < 10240);     // that long, tiles serve no zero point
    return M <= 16 || N <= 12288 || k_tiles(K) >= 16;
}

typedef hipError_t (*linear_fn)(const uint8_t *, const uint8_t *, int64_t, int64_t, int64_t, float, const float *,
                                const float *, int, const int32_t *, uint16_t *, int32_t *, hipStream_t);

static int linear_common(const char *fn, linear_fn force, const void *xq, const void *wq, int64_t M, int64_t N,
                         int64_t K, float s_a, const float *s_w, const float *d, int zp, const int32_t *wsum, void *y,
                         int32_t *acc, void *stream, void *workspace = nullptr, int64_t workspace_bytes = 0,
                         void *scratch = nullptr, int64_t scratch_bytes = 0)
{
    if (!xq || !wq || !s_w || !y) {
        set_error("%s: NULL pointer", fn);
        return FPTQ_ERR_NULL;
    }
    int rc;
    if ((rc = check_dims(fn, M, K, "M", "K")) || (rc = check_dims(fn, N, K, "N", "K")) ||
        (rc = check_dims(fn, M, N, "M", "N")))
        return rc;
    if (!(s_a > 0.0f) || !std::isfinite(s_a)) {
        set_error("%s: s_a must be finite and > 0", fn);
        return FPTQ_ERR_VALUE;
    }
    if ((rc = check_align(fn, xq, 16, "xq_packed")) || (rc = check_align(fn, wq, 16, "w_packed")) ||
        (rc = check_align(fn, y, 16, "y_bf16")) || (rc = check_align(fn, acc, 16, "acc_dbg")) ||
        (rc = check_align(fn, s_w, 4, "s_w")) || (rc = check_align(fn, d, 4, "row_out_scale")) ||
        (rc = check_align(fn, wsum, 4, "w_row_sum")))
        return rc;
    if (zp < -8 || zp > 7 || (zp != 0 && !wsum)) {
        set_error("%s: zero_point must be in [-8, 7] and needs w_row_sum", fn);
        return FPTQ_ERR_VALUE;
    }
    if (K > (zp != 0 ? MAX_K_ZERO_POINT : MAX_K)) {
        set_error("%s: K=%lld exceeds %lld, the longest sum INT32 holds exactly%s", fn, (long long)K,
                  (long long)(zp != 0 ? MAX_K_ZERO_POINT : MAX_K), zp != 0 ? " with a zero point" : "");
        return FPTQ_ERR_SHAPE;
    }
    if (zp == 0) wsum = nullptr;
    if ((rc = check_align(fn, workspace, 256, "workspace"))) return rc;
    if (workspace_bytes < 0) {
        set_error("%s: negative workspace_bytes", fn);
        return FPTQ_ERR_SIZE;
    }
    if ((rc = check_align(fn, scratch, 256, "scratch"))) return rc;
    if (scratch_bytes < 0) {
        set_error("%s: negative scratch_bytes", fn);
        return FPTQ_ERR_SIZE;
    }
    linear_fn f = force ? force : (few_token_shape(M, N, K) && forced_gemm_tile() == 0 ? launch_linear_decode : launch_linear_mfma);
    hipError_t e;
    const int tile_tokens = f == launch_linear_mfma && scratch ? prefill_tile(M, N, K) : 0;
    if (tile_tokens && scratch_bytes >= prefill_scratch_bytes(M, K))
        e = launch_linear_prefill((const uint8_t *)xq, (const uint8_t *)wq, M, N, K, s_a, s_w, d, zp, wsum, (uint16_t *)y, acc,
                                  (uint8_t *)scratch, tile_tokens, (hipStream_t)stream);
    else if (f == launch_linear_mfma && workspace)
        e = launch_linear_mfma_ws((const uint8_t *)xq, (const uint8_t *)wq, M, N, K, s_a, s_w, d, zp, wsum, (uint16_t *)y, acc,
                                  (int32_t *)workspace, workspace_bytes, (hipStream_t)stream);
    else
        e = f((const uint8_t *)xq, (const uint8_t *)wq, M, N, K, s_a, s_w, d, zp, wsum, (uint16_t *)y, acc, (hipStream_t)stream);
    return e == hipSuccess ? FPTQ_OK : hip_fail(fn, e);
}

// ---- attention: what its entry points check alike

static const int64_t MAX_TOKENS = (int64_t)1 << 24, MAX_STRIDE = (int64_t)1 << 24, MAX_HEADS = 4096;

static int check_heads(const char *fn, const fptq_heads *x, const char *name)
{
    if (!x || !x->data) {
        set_error("%s: NULL pointer (%s)", fn, name);
        return FPTQ_ERR_NULL;
    }
    for (int64_t stride : {x->token_stride, x->head_stride}) {
        if (stride < 0 || stride >= MAX_STRIDE) {
            set_error("%s: %s has a stride of %lld values, 0 to 2^24 - 8 are served", fn, name, (long long)stride);
            return FPTQ_ERR_SHAPE;
        }
        if (stride % 8) {
            set_error("%s: the strides of %s must be multiples of 8 values", fn, name);
            return FPTQ_ERR_ALIGN;
        }
    }
    return check_align(fn, x->data, 16, name);
}

static int check_attention(const char *fn, int64_t tokens, int64_t sequences, int heads, int kv_heads, int head_dim)
{
    if (tokens < 0 || tokens > MAX_TOKENS || sequences < 1 || sequences > MAX_TOKENS || heads < 1 || heads > MAX_HEADS || kv_heads < 1 || heads % kv_heads) {
        set_error("%s: bad shape tokens=%lld sequences=%lld heads=%d kv_heads=%d", fn, (long long)tokens, (long long)sequences, heads, kv_heads);
        return FPTQ_ERR_SHAPE;
    }
    if (head_dim != 64 && head_dim != 128) {
        set_error("%s: head_dim must be 64 or 128 (got %d)", fn, head_dim);
        return FPTQ_ERR_SHAPE;
    }
    return FPTQ_OK;
}

static int check_cache(const char *fn, const fptq_cache *c, int kv_heads, int head_dim, const int32_t *table, int64_t table_width, const int32_t *lengths,
                       const int32_t *cu, int64_t tokens, int64_t sequences)
{
    if (!c || !c->key_codes || !c->value_codes || !c->key_scales || !c->value_scales || !table || !lengths) {
        set_error("%s: NULL pointer (cache, table or lengths)", fn);
        return FPTQ_ERR_NULL;
    }
    if (c->pages < 1 || c->pages > 0x7fffffff || c->pages > MAX_ELEMS / ((int64_t)kv_heads * PAGE * head_dim) || table_width < 1 || table_width > 1 << 24) {
        set_error("%s: bad shape pages=%lld table_width=%lld", fn, (long long)c->pages, (long long)table_width);
        return FPTQ_ERR_SHAPE;
    }
    if (!cu && tokens != sequences) {
        set_error("%s: without cu every sequence has one token (%lld tokens, %lld sequences)", fn, (long long)tokens, (long long)sequences);
        return FPTQ_ERR_SHAPE;
    }
    int rc;
    if ((rc = check_align(fn, c->key_codes, 16, "key_codes")) || (rc = check_align(fn, c->value_codes, 16, "value_codes")) ||
        (rc = check_align(fn, c->key_scales, 4, "key_scales")) || (rc = check_align(fn, c->value_scales, 4, "value_scales")) ||
        (rc = check_align(fn, table, 4, "table")) || (rc = check_align(fn, lengths, 4, "lengths")) || (rc = check_align(fn, cu, 4, "cu")))
        return rc;
    return FPTQ_OK;
}

static int check_scale(const char *fn, float scale)
{
    if (!(scale > 0.0f) || !std::isfinite(scale)) {
        set_error("%s: scale must be finite and > 0", fn);
        return FPTQ_ERR_VALUE;
    }
    return FPTQ_OK;
}

static Heads heads_of(const fptq_heads *x) { return {(const uint16_t *)x->data, x->token_stride, x->head_stride}; }
static Cache cache_of(const fptq_cache *c) { return {(uint8_t *)c->key_codes, (uint8_t *)c->value_codes, c->key_scales, c->value_scales, c->pages}; }

// a launch that would have more workgroups than a grid may
static int launched(const char *fn, hipError_t e)
{
    if (e == hipErrorInvalidConfiguration) {
        set_error("%s: too many tokens, sequences and heads for one call", fn);
        return FPTQ_ERR_SHAPE;
    }
    return e == hipSuccess ? FPTQ_OK : hip_fail(fn, e);
}

}  // namespace fptq

using namespace fptq;

extern "C" {

int fptq_version(void) { return 210; }

int fptq_init(void)
{
    const DeviceInfo *info;
    hipError_t e = device_info(&info);
    return e == hipSuccess ? FPTQ_OK : hip_fail("fptq_init", e);
}

const char *fptq_last_error(void) { return g_err; }

int64_t fptq_packed_bytes(int64_t rows, int64_t K)
{
    if (check_dims("fptq_packed_bytes", rows, K, "rows", "K")) return FPTQ_ERR_SHAPE;
    return packed_bytes(rows, K);
}

int fptq_pack_weights(const int8_t *w_int, int64_t N, int64_t K, void *w_packed, int64_t w_packed_bytes, void *stream)
{
    if (!w_int || !w_packed) {
        set_error("fptq_pack_weights: NULL pointer");
        return FPTQ_ERR_NULL;
    }
    int rc = check_dims("fptq_pack_weights", N, K, "N", "K");
    if (rc) return rc;
    if (w_packed_bytes < packed_bytes(N, K)) {
        set_error("fptq_pack_weights: buffer of %lld bytes, need %lld", (long long)w_packed_bytes,
                  (long long)packed_bytes(N, K));
        return FPTQ_ERR_SIZE;
    }
    if ((rc = check_align("fptq_pack_weights", w_packed, 16, "w_packed"))) return rc;
    hipError_t e = launch_pack_weights(w_int, N, K, (uint8_t *)w_packed, (hipStream_t)stream);
    return e == hipSuccess ? FPTQ_OK : hip_fail("fptq_pack_weights", e);
}

static int quantize_common(const char *fn, int hadamard_block, int zero_point, const void *x_bf16, int64_t M, int64_t K, int scale_mode,
                           float eps, const float *row_scale_in, float s_a, void *xq_packed, int64_t xq_bytes,
                           float *row_scale_out, void *stream)
{
    if (!x_bf16 || !xq_packed) {
        set_error("%s: NULL pointer", fn);
        return FPTQ_ERR_NULL;
    }
    int rc = check_dims(fn, M, K, "M", "K");
    if (rc) return rc;
    const bool block_ok = hadamard_block == 256 || hadamard_block == 512 || hadamard_block == 1024 || hadamard_block == 2048 ||
                          hadamard_block == 4096;
    if (hadamard_block != 0 && (!block_ok || K % hadamard_block != 0)) {
        set_error("%s: hadamard_block must be 256, 512, 1024, 2048 or 4096 and divide K (got block %d, K %lld)", fn, hadamard_block,
                  (long long)K);
        return FPTQ_ERR_SHAPE;
    }
    if (scale_mode != FPTQ_SCALE_NONE && scale_mode != FPTQ_SCALE_RMS && scale_mode != FPTQ_SCALE_GIVEN) {
        set_error("%s: unknown scale_mode %d", fn, scale_mode);
        return FPTQ_ERR_MODE;
    }
    if (scale_mode == FPTQ_SCALE_GIVEN && !row_scale_in) {
        set_error("%s: FPTQ_SCALE_GIVEN needs row_scale_in", fn);
        return FPTQ_ERR_MODE;
    }
    if (!(s_a > 0.0f) || !std::isfinite(s_a) || !(eps >= 0.0f) || zero_point < -8 || zero_point > 7) {
        set_error("%s: s_a must be finite and > 0, eps >= 0, zero_point in [-8, 7]", fn);
        return FPTQ_ERR_VALUE;
    }
    if (xq_bytes < packed_bytes(M, K)) {
        set_error("%s: buffer of %lld bytes, need %lld", fn, (long long)xq_bytes, (long long)packed_bytes(M, K));
        return FPTQ_ERR_SIZE;
    }
    if ((rc = check_align(fn, xq_packed, 16, "xq_packed")) || (rc = check_align(fn, x_bf16, hadamard_block ? 16 : 2, "x_bf16")) ||
        (rc = check_align(fn, row_scale_in, 4, "row_scale_in")) || (rc = check_align(fn, row_scale_out, 4, "row_scale_out")))
        return rc;
    // the one fp32 division of the quantizer happens here, on the host
    volatile float inv = 1.0f / s_a;
    hipError_t e = hadamard_block
                       ? launch_quantize_act_hadamard((const uint16_t *)x_bf16, M, K, hadamard_block, scale_mode, eps, row_scale_in, inv,
                                                      (uint8_t *)xq_packed, row_scale_out, (hipStream_t)stream)
                       : launch_quantize_act((const uint16_t *)x_bf16, M, K, scale_mode, eps, row_scale_in, inv, zero_point,
                                             (uint8_t *)xq_packed, row_scale_out, (hipStream_t)stream);
    return e == hipSuccess ? FPTQ_OK : hip_fail(fn, e);
}

int fptq_quantize_act(const void *x_bf16, int64_t M, int64_t K, int scale_mode, float eps, const float *row_scale_in,
                      float s_a, void *xq_packed, int64_t xq_bytes, float *row_scale_out, void *stream)
{
    return quantize_common("fptq_quantize_act", 0, 0, x_bf16, M, K, scale_mode, eps, row_scale_in, s_a, xq_packed, xq_bytes,
                           row_scale_out, stream);
}

int fptq_quantize_act_asym(const void *x_bf16, int64_t M, int64_t K, int scale_mode, float eps, const float *row_scale_in,
                           float s_a, int zero_point, void *xq_packed, int64_t xq_bytes, float *row_scale_out, void *stream)
{
    return quantize_common("fptq_quantize_act_asym", 0, zero_point, x_bf16, M, K, scale_mode, eps, row_scale_in, s_a, xq_packed,
                           xq_bytes, row_scale_out, stream);
}

int fptq_residual_norm_quantize(const void *x_res_bf16, const void *y_bf16, int64_t M, int64_t K, const float *s_prev,
                                float eps, float s_a, void *x_next_bf16, float *s_next, void *xq_packed, int64_t xq_bytes,
                                void *stream)
{
    const char *fn = "fptq_residual_norm_quantize";
    if (!x_res_bf16 || !y_bf16 || !x_next_bf16 || !s_next || !xq_packed) {
        set_error("%s: NULL pointer", fn);
        return FPTQ_ERR_NULL;
    }
    int rc = check_dims(fn, M, K, "M", "K");
    if (rc) return rc;
    if (!(s_a > 0.0f) || !std::isfinite(s_a) || !(eps >= 0.0f)) {
        set_error("%s: s_a must be finite and > 0, eps >= 0", fn);
        return FPTQ_ERR_VALUE;
    }
    if (xq_bytes < packed_bytes(M, K)) {
        set_error("%s: buffer of %lld bytes, need %lld", fn, (long long)xq_bytes, (long long)packed_bytes(M, K));
        return FPTQ_ERR_SIZE;
    }
    if ((rc = check_align(fn, xq_packed, 16, "xq_packed")) || (rc = check_align(fn, x_res_bf16, 2, "x_res_bf16")) ||
        (rc = check_align(fn, y_bf16, 2, "y_bf16")) || (rc = check_align(fn, x_next_bf16, 2, "x_next_bf16")) ||
        (rc = check_align(fn, s_prev, 4, "s_prev")) || (rc = check_align(fn, s_next, 4, "s_next")))
        return rc;
    volatile float inv = 1.0f / s_a;
    hipError_t e = launch_residual_norm_quantize((const uint16_t *)x_res_bf16, (const uint16_t *)y_bf16, M, K, s_prev, eps, inv,
                                                 (uint16_t *)x_next_bf16, s_next, (uint8_t *)xq_packed, (hipStream_t)stream);
    return e == hipSuccess ? FPTQ_OK : hip_fail(fn, e);
}

int fptq_quantize_act_dynamic(const void *x_bf16, int64_t M, int64_t K, void *xq_packed, int64_t xq_bytes,
                              float *token_scale_out, void *stream)
{
    const char *fn = "fptq_quantize_act_dynamic";
    if (!x_bf16 || !xq_packed || !token_scale_out) {
        set_error("%s: NULL pointer", fn);
        return FPTQ_ERR_NULL;
    }
    int rc = check_dims(fn, M, K, "M", "K");
    if (rc) return rc;
    if (xq_bytes < packed_bytes(M, K)) {
        set_error("%s: buffer of %lld bytes, need %lld", fn, (long long)xq_bytes, (long long)packed_bytes(M, K));
        return FPTQ_ERR_SIZE;
    }
    if ((rc = check_align(fn, xq_packed, 16, "xq_packed")) || (rc = check_align(fn, x_bf16, 2, "x_bf16")) ||
        (rc = check_align(fn, token_scale_out, 4, "token_scale_out")))
        return rc;
    hipError_t e = launch_quantize_act_dynamic((const uint16_t *)x_bf16, M, K, (uint8_t *)xq_packed, token_scale_out,
                                               (hipStream_t)stream);
    return e == hipSuccess ? FPTQ_OK : hip_fail(fn, e);
}

int fptq_quantize_act_hadamard(const void *x_bf16, int64_t M, int64_t K, int hadamard_block, int scale_mode, float eps,
                               const float *row_scale_in, float s_a, void *xq_packed, int64_t xq_bytes,
                               float *row_scale_out, void *stream)
{
    if (hadamard_block == 0) {
        set_error("fptq_quantize_act_hadamard: hadamard_block must be 256, 512, 1024, 2048 or 4096");
        return FPTQ_ERR_SHAPE;
    }
    return quantize_common("fptq_quantize_act_hadamard", hadamard_block, 0, x_bf16, M, K, scale_mode, eps, row_scale_in, s_a,
                           xq_packed, xq_bytes, row_scale_out, stream);
}

int fptq_w4a4_linear(const void *xq_packed, const void *w_packed, int64_t M, int64_t N, int64_t K, float s_a,
                     const float *s_w, const float *row_out_scale, void *y_bf16, int32_t *acc_dbg, void *stream)
{
    return linear_common("fptq_w4a4_linear", nullptr, xq_packed, w_packed, M, N, K, s_a, s_w, row_out_scale, 0, nullptr,
                         y_bf16, acc_dbg, stream);
}

int fptq_w4a4_linear_zp(const void *xq_packed, const void *w_packed, int64_t M, int64_t N, int64_t K, float s_a,
                        const float *s_w, const float *row_out_scale, int zero_point, const int32_t *w_row_sum,
                        void *y_bf16, int32_t *acc_dbg, void *stream)
{
    return linear_common("fptq_w4a4_linear_zp", nullptr, xq_packed, w_packed, M, N, K, s_a, s_w, row_out_scale, zero_point,
                         w_row_sum, y_bf16, acc_dbg, stream);
}

int fptq_weight_row_sums(const int8_t *w_int, int64_t N, int64_t K, int32_t *sums, void *stream)
{
    if (!w_int || !sums) {
        set_error("fptq_weight_row_sums: NULL pointer");
        return FPTQ_ERR_NULL;
    }
    int rc = check_dims("fptq_weight_row_sums", N, K, "N", "K");
    if (rc) return rc;
    if ((rc = check_align("fptq_weight_row_sums", sums, 4, "sums"))) return rc;
    hipError_t e = launch_weight_row_sums(w_int, N, K, sums, (hipStream_t)stream);
    return e == hipSuccess ? FPTQ_OK : hip_fail("fptq_weight_row_sums", e);
}

int fptq_w4a4_linear_ref(const void *xq_packed, const void *w_packed, int64_t M, int64_t N, int64_t K, float s_a,
                         const float *s_w, const float *row_out_scale, void *y_bf16, int32_t *acc_dbg, void *stream)
{
    return linear_common("fptq_w4a4_linear_ref", launch_linear_ref, xq_packed, w_packed, M, N, K, s_a, s_w,
                         row_out_scale, 0, nullptr, y_bf16, acc_dbg, stream);
}

int64_t fptq_linear_workspace_bytes(int64_t M, int64_t N, int64_t K)
{
    const char *fn = "fptq_linear_workspace_bytes";
    int rc;
    if ((rc = check_dims(fn, M, K, "M", "K")) || (rc = check_dims(fn, N, K, "N", "K")) || (rc = check_dims(fn, M, N, "M", "N")))
        return rc;
    if (K > MAX_K) {
        set_error("%s: K=%lld exceeds %lld, the longest sum INT32 holds exactly", fn, (long long)K, (long long)MAX_K);
        return FPTQ_ERR_SHAPE;
    }
    return few_token_shape(M, N, K) ? 0 : linear_workspace_bytes(M, N, K);
}

int fptq_w4a4_linear_ws(const void *xq_packed, const void *w_packed, int64_t M, int64_t N, int64_t K, float s_a,
                        const float *s_w, const float *row_out_scale, void *y_bf16, int32_t *acc_dbg, void *workspace,
                        int64_t workspace_bytes, void *stream)
{
    return linear_common("fptq_w4a4_linear_ws", nullptr, xq_packed, w_packed, M, N, K, s_a, s_w, row_out_scale, 0, nullptr, y_bf16,
                         acc_dbg, stream, workspace, workspace_bytes);
}

int fptq_w4a4_linear_noalloc(const void *xq_packed, const void *w_packed, int64_t M, int64_t N, int64_t K, float s_a,
                             const float *s_w, const float *row_out_scale, void *y_bf16, int32_t *acc_dbg, void *stream)
{
    const char *fn = "fptq_w4a4_linear_noalloc";
    // shapes that would not split K anyway need no scratch: the plain layer (which allocates nothing either)
    const int64_t need = (M >= 1 && N >= 1 && K >= 1 && K <= MAX_K && M <= MAX_ELEMS / K && N <= MAX_ELEMS / K && M <= MAX_ELEMS / N &&
                          !few_token_shape(M, N, K))
                             ? linear_workspace_bytes(M, N, K)
                             : 0;
    if (need == 0)
        return linear_common(fn, nullptr, xq_packed, w_packed, M, N, K, s_a, s_w, row_out_scale, 0, nullptr, y_bf16, acc_dbg, stream);
    const DeviceInfo *info;
    hipError_t e = device_info(&info);
    if (e != hipSuccess) return hip_fail(fn, e);
    if (need > info->scratch_bytes) {
        set_error("%s: M=%lld N=%lld K=%lld needs %lld bytes of scratch, the built-in area holds %lld; use fptq_w4a4_linear_ws "
                  "with a caller workspace or fptq_w4a4_linear", fn, (long long)M, (long long)N, (long long)K, (long long)need,
                  (long long)info->scratch_bytes);
        return FPTQ_ERR_SIZE;
    }
    return linear_common(fn, nullptr, xq_packed, w_packed, M, N, K, s_a, s_w, row_out_scale, 0, nullptr, y_bf16, acc_dbg, stream,
                         info->scratch, info->scratch_bytes);
}

int64_t fptq_linear_scratch_bytes(int64_t M, int64_t N, int64_t K)
{
    const char *fn = "fptq_linear_scratch_bytes";
    int rc;
    if ((rc = check_dims(fn, M, K, "M", "K")) || (rc = check_dims(fn, N, K, "N", "K")) || (rc = check_dims(fn, M, N, "M", "N")))
        return rc;
    if (K > MAX_K) {
        set_error("%s: K=%lld exceeds %lld, the longest sum INT32 holds exactly", fn, (long long)K, (long long)MAX_K);
        return FPTQ_ERR_SHAPE;
    }
    return !few_token_shape(M, N, K) && prefill_tile(M, N, K) ? prefill_scratch_bytes(M, K) : 0;
}

int fptq_w4a4_linear_scratch(const void *xq_packed, const void *w_packed, int64_t M, int64_t N, int64_t K, float s_a,
                             const float *s_w, const float *row_out_scale, int zero_point, const int32_t *w_row_sum, void *y_bf16,
                             int32_t *acc_dbg, void *scratch, int64_t scratch_bytes, void *stream)
{
    return linear_common("fptq_w4a4_linear_scratch", nullptr, xq_packed, w_packed, M, N, K, s_a, s_w, row_out_scale, zero_point,
                         w_row_sum, y_bf16, acc_dbg, stream, nullptr, 0, scratch, scratch_bytes);
}

int fptq_linear_launch_plan(int64_t M, int64_t N, int64_t K, int with_workspace, char *kernel, int kernel_len,
                            int64_t *workgroups, int *threads)
{
    const char *fn = "fptq_linear_launch_plan";
    if (!kernel || kernel_len < 1 || !workgroups || !threads) {
        set_error("%s: NULL pointer", fn);
        return FPTQ_ERR_NULL;
    }
    int rc;
    if ((rc = check_dims(fn, M, K, "M", "K")) || (rc = check_dims(fn, N, K, "N", "K")) || (rc = check_dims(fn, M, N, "M", "N")))
        return rc;
    LinearPlan plan = {};
    if (few_token_shape(M, N, K) && forced_gemm_tile() == 0) {
        snprintf(plan.kernel, sizeof plan.kernel, "linear_decode_kernel");
        plan.workgroups = 0;
        plan.threads = 0;
    } else if (const int tile_tokens = with_workspace == 2 ? prefill_tile(M, N, K) : 0) {
        snprintf(plan.kernel, sizeof plan.kernel, "linear_prefill_kernel");
        plan.workgroups = prefill_workgroups(M, N, tile_tokens);
        plan.threads = 256;
    } else {
        linear_mfma_plan(M, N, K, with_workspace == 1, &plan);
    }
    snprintf(kernel, (size_t)kernel_len, "%s", plan.kernel);
    *workgroups = plan.workgroups;
    *threads = plan.threads;
    return FPTQ_OK;
}

int fptq_set_gemm_map(int mode)
{
    if (mode != 0 && mode != 1) {
        set_error("fptq_set_gemm_map: mode must be 0 or 1");
        return FPTQ_ERR_VALUE;
    }
    set_gemm_map(mode);
    return FPTQ_OK;
}

int fptq_set_linear_prefill(int mode)
{
    if ((mode < 0 || mode > 2) && mode != 128 && mode != 192 && mode != 256) {
        set_error("fptq_set_linear_prefill: mode must be 0, 1, 2, 128, 192 or 256");
        return FPTQ_ERR_VALUE;
    }
    set_linear_prefill(mode);
    return FPTQ_OK;
}

int fptq_set_decode_shape(int code)
{
    if (!set_decode_shape(code)) {
        set_error("fptq_set_decode_shape: code must be 0 or waves (8, 16) * 100 + tiles per batch (1, 2, 4) * 10 + channel groups (1, 2, 4)");
        return FPTQ_ERR_VALUE;
    }
    return FPTQ_OK;
}

int fptq_set_gemm_tile(int tile)
{
    if (tile < 0 || tile > 8) {
        set_error("fptq_set_gemm_tile: tile must be 0..8");
        return FPTQ_ERR_VALUE;
    }
    set_gemm_tile(tile);
    return FPTQ_OK;
}

int fptq_cache_append(const fptq_heads *q, const fptq_heads *k, const fptq_heads *v, int64_t tokens, int64_t sequences, int heads, int kv_heads,
                      int head_dim, const float *rope, int64_t positions, int rope_dims, int interleaved, const fptq_cache *cache, const int32_t *table,
                      int64_t table_width, const int32_t *lengths, const int32_t *cu, void *q_out, void *k_out, void *stream)
{
    const char *fn = "fptq_cache_append";
    int rc;
    if ((rc = check_attention(fn, tokens, sequences, heads, kv_heads, head_dim))) return rc;
    if (tokens == 0) return FPTQ_OK;             // an empty tensor has no address
    if ((rc = check_heads(fn, q, "q")) || (rc = check_heads(fn, k, "k")) || (rc = check_heads(fn, v, "v")) ||
        (rc = check_cache(fn, cache, kv_heads, head_dim, table, table_width, lengths, cu, tokens, sequences)))
        return rc;
    if (!q_out || (rope_dims != 0 && !rope)) {
        set_error("%s: NULL pointer (%s)", fn, q_out ? "rope" : "q_out");
        return FPTQ_ERR_NULL;
    }
    if (rope_dims < 0 || rope_dims > head_dim || rope_dims % 16 || (rope_dims && (positions < 1 || positions > MAX_ELEMS / rope_dims))) {
        set_error("%s: rope_dims must be a multiple of 16 up to head_dim, positions >= 1 (got %d, %lld)", fn, rope_dims, (long long)positions);
        return FPTQ_ERR_SHAPE;
    }
    if ((rc = check_align(fn, rope, 16, "rope")) || (rc = check_align(fn, q_out, 16, "q_out")) || (rc = check_align(fn, k_out, 16, "k_out"))) return rc;
    const Sequences s = {cu, lengths, table, (int32_t)sequences, (int32_t)tokens, table_width};
    return launched(fn, launch_cache_append(heads_of(q), heads_of(k), heads_of(v), s, heads, kv_heads, head_dim, rope, positions, rope_dims, interleaved != 0,
                                            cache_of(cache), (uint16_t *)q_out, (uint16_t *)k_out, (hipStream_t)stream));
}

int64_t fptq_cached_attention_scratch_bytes(int64_t tokens, int64_t sequences, int heads, int kv_heads, int head_dim, int64_t table_width)
{
    const char *fn = "fptq_cached_attention_scratch_bytes";
    const int rc = check_attention(fn, tokens, sequences, heads, kv_heads, head_dim);
    if (rc) return rc;
    if (table_width < 1 || table_width > 1 << 24) {
        set_error("%s: bad shape table_width=%lld", fn, (long long)table_width);
        return FPTQ_ERR_SHAPE;
    }
    return cached_attention_scratch_bytes(tokens, sequences, heads, kv_heads, head_dim, table_width);
}

int fptq_cached_attention(const fptq_heads *q, int64_t tokens, int64_t sequences, int heads, int kv_heads, int head_dim, float scale,
                          const fptq_cache *cache, const int32_t *table, int64_t table_width, const int32_t *lengths, const int32_t *cu, void *out,
                          void *scratch, int64_t scratch_bytes, void *stream)
{
    const char *fn = "fptq_cached_attention";
    int rc;
    if ((rc = check_attention(fn, tokens, sequences, heads, kv_heads, head_dim))) return rc;
    if (tokens == 0) return FPTQ_OK;
    if ((rc = check_heads(fn, q, "q")) ||
        (rc = check_cache(fn, cache, kv_heads, head_dim, table, table_width, lengths, cu, tokens, sequences)) || (rc = check_scale(fn, scale)))
        return rc;
    if (!out) {
        set_error("%s: NULL pointer (out)", fn);
        return FPTQ_ERR_NULL;
    }
    if (scratch_bytes < 0) {
        set_error("%s: negative scratch_bytes", fn);
        return FPTQ_ERR_SIZE;
    }
    if ((rc = check_align(fn, out, 16, "out")) || (rc = check_align(fn, scratch, 256, "scratch"))) return rc;
    const Sequences s = {cu, lengths, table, (int32_t)sequences, (int32_t)tokens, table_width};
    return launched(fn, launch_cached_attention(heads_of(q), s, heads, kv_heads, head_dim, scale, cache_of(cache), (uint16_t *)out, (uint8_t *)scratch,
                                                scratch_bytes, (hipStream_t)stream));
}

int fptq_prompt_attention(const fptq_heads *q, const fptq_heads *k, const fptq_heads *v, int64_t tokens, int64_t sequences, int heads, int kv_heads,
                          int head_dim, float scale, const int32_t *cu, void *out, void *stream)
{
    const char *fn = "fptq_prompt_attention";
    int rc;
    if ((rc = check_attention(fn, tokens, sequences, heads, kv_heads, head_dim))) return rc;
    if (tokens == 0) return FPTQ_OK;
    if ((rc = check_heads(fn, q, "q")) || (rc = check_heads(fn, k, "k")) ||
        (rc = check_heads(fn, v, "v")) || (rc = check_scale(fn, scale)))
        return rc;
    if (!cu || !out) {
        set_error("%s: NULL pointer (%s)", fn, cu ? "out" : "cu");
        return FPTQ_ERR_NULL;
    }
    if ((rc = check_align(fn, cu, 4, "cu")) || (rc = check_align(fn, out, 16, "out"))) return rc;
    const Sequences s = {cu, nullptr, nullptr, (int32_t)sequences, (int32_t)tokens, 0};
    return launched(fn, launch_prompt_attention(heads_of(q), heads_of(k), heads_of(v), s, heads, kv_heads, head_dim, scale, (uint16_t *)out,
                                                (hipStream_t)stream));
}

int fptq_unpack(const void *packed, int64_t rows, int64_t K, int8_t *out_int8, void *stream)
{
    if (!packed || !out_int8) {
        set_error("fptq_unpack: NULL pointer");
        return FPTQ_ERR_NULL;
    }
    int rc = check_dims("fptq_unpack", rows, K, "rows", "K");
    if (rc) return rc;
    if ((rc = check_align("fptq_unpack", packed, 16, "packed"))) return rc;
    hipError_t e = launch_unpack((const uint8_t *)packed, rows, K, out_int8, (hipStream_t)stream);
    return e == hipSuccess ? FPTQ_OK : hip_fail("fptq_unpack", e);
}

}  // extern "C"
