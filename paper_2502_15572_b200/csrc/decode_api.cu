// C ABI of the decoding step's operators that need no handle: dresd_drafts_sample (k13_sample.cu) and the products with 4-bit
// weights (k15_w4.cu).  Argument validation only.
#include <atomic>
#include <cstring>
#include <map>
#include <new>

#include "api_util.h"

using namespace dresd;

namespace {

constexpr int kMaxVocab = 1 << 20;
constexpr long long kMaxDistance = 1LL << 38;

// process-wide, for tests (dresd_set_global_option)
std::atomic<int> g_w4_path{0}, g_w4_wait_ms{0}, g_w4_lose_stage{0};

dresd_status current_device(int *dev, int *sms)
{
    cudaError_t e = cudaGetDevice(dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, *dev);
    return e == cudaSuccess ? DRESD_OK : fail_cuda(e, "device query");
}

dresd_status check_w4(int inputs, int outputs, dresd_dtype dtype, int group)
{
    if (dtype != DRESD_F32 && dtype != DRESD_F16 && dtype != DRESD_BF16) return fail(DRESD_ERR_INVALID, "unknown dtype %d", (int)dtype);
    if (dtype == DRESD_F32) return fail(DRESD_ERR_UNSUPPORTED, "4-bit weights go with fp16 or bf16");
    if (inputs < 1 || outputs < 1 || group < 1) return fail(DRESD_ERR_INVALID, "inputs = %d, outputs = %d, group = %d", inputs, outputs, group);
    if (group != 32 && group != 64 && group != 128) return fail(DRESD_ERR_UNSUPPORTED, "group = %d is not 32, 64 or 128", group);
    if (inputs % group != 0) return fail(DRESD_ERR_INVALID, "inputs = %d is not a multiple of group = %d", inputs, group);
    if (inputs > DRESD_MAX_W4_SIZE || outputs > DRESD_MAX_W4_SIZE)
        return fail(DRESD_ERR_UNSUPPORTED, "inputs = %d / outputs = %d exceed %d", inputs, outputs, DRESD_MAX_W4_SIZE);
    return DRESD_OK;
}

}  // namespace

extern "C" {

dresd_status dresd_drafts_sample(const void *logits, dresd_dtype dtype, int64_t chunk_stride, int64_t row_stride, int V,
                                 const int32_t *drafts, const int32_t *valid, const float *uniform, const float *temperature,
                                 const int32_t *top_k, const float *top_p, int B, int n, int L, int32_t *out_best,
                                 int32_t *out_len, int32_t *out_tokens, float *out_logprobs, void *stream)
{
    if (dtype != DRESD_F32 && dtype != DRESD_F16 && dtype != DRESD_BF16) return fail(DRESD_ERR_INVALID, "unknown dtype %d", (int)dtype);
    if (B < 0 || V < 1) return fail(DRESD_ERR_INVALID, "B = %d, V = %d", B, V);
    if (n < 0 || L < 0 || (n == 0) != (L == 0)) return fail(DRESD_ERR_INVALID, "n = %d, L = %d", n, L);
    if (n > DRESD_MAX_TOP_N) return fail(DRESD_ERR_UNSUPPORTED, "n = %d exceeds DRESD_MAX_TOP_N", n);
    if (L > 65536) return fail(DRESD_ERR_UNSUPPORTED, "L = %d exceeds 65536", L);
    if (V > kMaxVocab) return fail(DRESD_ERR_UNSUPPORTED, "V = %d exceeds %d", V, kMaxVocab);
    if (B > 65535) return fail(DRESD_ERR_UNSUPPORTED, "B = %d exceeds 65535", B);
    if (n > 0 && (row_stride < V || row_stride >= kMaxDistance)) return fail(DRESD_ERR_INVALID, "rows of %d logits lie %lld apart", V, (long long)row_stride);
    if (B > 1 && (chunk_stride < V || chunk_stride >= kMaxDistance))
        return fail(DRESD_ERR_INVALID, "chunks of %d logits a row lie %lld apart", V, (long long)chunk_stride);
    if (B == 0) return DRESD_OK;
    int dev = -1, sms = 0;
    const dresd_status st = current_device(&dev, &sms);
    if (st != DRESD_OK) return st;
    if (!is_device_ptr(logits, dev) || !aligned(logits, dtype == DRESD_F32 ? 4 : 2))
        return fail(DRESD_ERR_INVALID, "logits must be an aligned pointer of the current device");
    if (n > 0 && (!is_word_ptr(drafts, dev) || !is_word_ptr(valid, dev)))
        return fail(DRESD_ERR_INVALID, "drafts/valid must be 4-byte aligned pointers of the current device");
    if (!is_word_ptr(uniform, dev) || (temperature && !is_word_ptr(temperature, dev)) || (top_k && !is_word_ptr(top_k, dev)) ||
        (top_p && !is_word_ptr(top_p, dev)))
        return fail(DRESD_ERR_INVALID, "uniform/temperature/top_k/top_p must be 4-byte aligned pointers of the current device (the last three may be NULL)");
    if (!is_word_ptr(out_best, dev) || !is_word_ptr(out_len, dev) || !is_word_ptr(out_tokens, dev) ||
        (out_logprobs && !is_word_ptr(out_logprobs, dev)))
        return fail(DRESD_ERR_INVALID, "out_* must be 4-byte aligned pointers of the current device (out_logprobs may be NULL)");
    SampleArgs a{};
    a.logits = logits;
    a.chunk_stride = chunk_stride;
    a.row_stride = row_stride;
    a.drafts = drafts;
    a.valid = valid;
    a.uniform = uniform;
    a.temperature = temperature;
    a.top_p = top_p;
    a.top_k = top_k;
    a.B = B;
    a.n = n;
    a.L = L;
    a.V = V;
    a.out_best = out_best;
    a.out_len = out_len;
    a.out_tokens = out_tokens;
    a.out_logs = out_logprobs;
    const cudaError_t e = launch_sample(a, (int)dtype, sms, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? DRESD_OK : fail_cuda(e, "drafts_sample launch");
}

dresd_status dresd_w4_quantise(const void *w, int64_t w_in, int64_t w_out, int inputs, int outputs, dresd_dtype dtype, int group,
                               uint8_t *out_codes, void *out_scales, void *stream)
{
    dresd_status st = check_w4(inputs, outputs, dtype, group);
    if (st != DRESD_OK) return st;
    if (w_in < 1 || w_out < 1 || w_in >= kMaxDistance || w_out >= kMaxDistance)
        return fail(DRESD_ERR_INVALID, "inputs lie %lld and outputs %lld elements apart", (long long)w_in, (long long)w_out);
    int dev = -1, sms = 0;
    if ((st = current_device(&dev, &sms)) != DRESD_OK) return st;
    if (!is_device_ptr(w, dev) || !aligned(w, 2)) return fail(DRESD_ERR_INVALID, "w must be an aligned pointer of the current device");
    if (!is_device_ptr(out_codes, dev) || !is_device_ptr(out_scales, dev) || !aligned(out_codes, 16) || !aligned(out_scales, 2))
        return fail(DRESD_ERR_INVALID, "out_codes (16-byte aligned) and out_scales must be pointers of the current device");
    const cudaError_t e = launch_w4_quantise(w, w_in, w_out, inputs, outputs, (int)dtype, group, out_codes, out_scales, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? DRESD_OK : fail_cuda(e, "w4_quantise launch");
}

dresd_status dresd_w4_matmul(const void *x, int64_t x_row, int rows, const uint8_t *codes, const void *scales, int inputs, int outputs,
                             dresd_dtype dtype, int group, int relu, const void *residual, int64_t residual_row, void *out,
                             int64_t out_row, void *stream)
{
    dresd_status st = check_w4(inputs, outputs, dtype, group);
    if (st != DRESD_OK) return st;
    if (rows < 0) return fail(DRESD_ERR_INVALID, "rows = %d is negative", rows);
    if (rows > DRESD_MAX_W4_SIZE) return fail(DRESD_ERR_UNSUPPORTED, "rows = %d exceed %d", rows, DRESD_MAX_W4_SIZE);
    if (rows > 1 && (x_row < inputs || x_row % 8 != 0 || x_row >= kMaxDistance))
        return fail(DRESD_ERR_INVALID, "x: rows of %d elements lie %lld apart; that has to be a multiple of 8", inputs, (long long)x_row);
    if (rows > 1 && (out_row < outputs || out_row >= kMaxDistance || (residual && (residual_row < outputs || residual_row >= kMaxDistance))))
        return fail(DRESD_ERR_INVALID, "out/residual: rows of %d elements lie %lld/%lld apart", outputs, (long long)out_row, (long long)residual_row);
    if (rows == 0) return DRESD_OK;
    int dev = -1, sms = 0;
    if ((st = current_device(&dev, &sms)) != DRESD_OK) return st;
    if (!is_device_ptr(x, dev) || !aligned(x, 16)) return fail(DRESD_ERR_INVALID, "x must be a 16-byte aligned pointer of the current device");
    if (!is_device_ptr(codes, dev) || !is_device_ptr(scales, dev) || !aligned(codes, 16) || !aligned(scales, 2))
        return fail(DRESD_ERR_INVALID, "codes (16-byte aligned) and scales must be pointers of the current device");
    if (!is_device_ptr(out, dev) || !aligned(out, 2) || (residual && (!is_device_ptr(residual, dev) || !aligned(residual, 2))))
        return fail(DRESD_ERR_INVALID, "out and residual (which may be NULL) must be aligned pointers of the current device");
    W4Args a{};
    a.x = x;
    a.x_row = x_row;
    a.codes = codes;
    a.scales = scales;
    a.residual = residual;
    a.residual_row = residual_row;
    a.out = out;
    a.out_row = out_row;
    a.rows = rows;
    a.inputs = inputs;
    a.outputs = outputs;
    a.groups = inputs / group;
    a.relu = relu != 0;
    cudaError_t e;
    const int path = g_w4_path.load();
    // Up to 16 rows mma.sync keeps up with the weights (4096 x 11008: 16.6 us, tcgen05 15.5; 11008 x 4096: 13.8 and 21; 4096 x 4096: 8.1 and 10.9).  Beyond, it
    // takes a step for every 32 rows and tcgen05 one for 128, at a fixed cost of some 5 us more, which is what 30 million weights take a step (4096 x 4096:
    // 32 rows 9.9 and 12.3 us, 48 rows 19.8 and 12.8; 2048 x 512: 256 rows 8.0 and 12.3; 4096 x 11008: 32 rows 27 and 16.5).
    const bool many = rows > 16 && (long long)inputs * outputs * ((rows + 31) / 32) > 30000000;
    if (path == 0 ? many : path == 2) {
        CUtensorMap code_map, x_map;
        const cuuint64_t code_dims[2] = {(cuuint64_t)inputs / 2, (cuuint64_t)outputs}, code_strides[1] = {(cuuint64_t)inputs / 2};
        // the distance of a single row is never used, but has to be a valid one
        const cuuint64_t x_dims[2] = {(cuuint64_t)inputs, (cuuint64_t)rows}, x_strides[1] = {(cuuint64_t)(rows > 1 ? x_row : inputs) * 2};
        const cuuint32_t code_box[2] = {64, 256}, x_box[2] = {64, (cuuint32_t)w4_umma_rows(rows)};
        if (!encode(&code_map, codes, kE4M3, 2, code_dims, code_strides, code_box, CU_TENSOR_MAP_SWIZZLE_64B) ||
            !encode(&x_map, x, (int)dtype, 2, x_dims, x_strides, x_box))
            return fail(DRESD_ERR_CUDA, "cuTensorMapEncodeTiled failed");
        const int ms = g_w4_wait_ms.load();
        e = launch_w4_umma(code_map, x_map, a, (int)dtype, group, ms > 0 ? ms * 2000000LL : 4000000000LL, g_w4_lose_stage.load(), sms,
                           static_cast<cudaStream_t>(stream));
    } else {
        e = launch_w4_matmul(a, (int)dtype, group, static_cast<cudaStream_t>(stream));
    }
    return e == cudaSuccess ? DRESD_OK : fail_cuda(e, "w4_matmul launch");
}

dresd_status dresd_w4_status(void *stream)
{
    // The device counts and never forgets; every thread has its own mark, by device.  (A word that is read and cleared would lose what
    // another stream reports between the two, and a report taken by one thread would be missing for the next.)
    static thread_local std::map<int, unsigned int> told;
    unsigned int count = 0;
    int dev = -1;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = w4_expired(&count, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return fail_cuda(e, "status read");
    try {
        unsigned int &mark = told[dev];
        if (mark == count) return DRESD_OK;
        mark = count;
    } catch (const std::bad_alloc &) {
        return fail(DRESD_ERR_ALLOC, "host allocation failed");
    }
    return fail(DRESD_ERR_TIMEOUT, "a device-side wait expired");
}

}  // extern "C"

namespace dresd {

int set_w4_option(const char *name, int value)
{
    if (std::strcmp(name, "w4_path") == 0) {
        if (value < 0 || value > 2) return fail(DRESD_ERR_INVALID, "w4_path = %d outside 0..2", value);
        g_w4_path.store(value);
    } else if (std::strcmp(name, "w4_wait_ms") == 0) {
        if (value < 0 || value > 60000) return fail(DRESD_ERR_INVALID, "w4_wait_ms = %d outside 0..60000", value);
        g_w4_wait_ms.store(value);
    } else if (std::strcmp(name, "w4_debug_lose_stage") == 0) {
        if (value < 0) return fail(DRESD_ERR_INVALID, "w4_debug_lose_stage = %d is negative", value);
        g_w4_lose_stage.store(value);
    } else {
        return fail(DRESD_ERR_INVALID, "unknown global option '%s'", name);
    }
    return DRESD_OK;
}

}  // namespace dresd
