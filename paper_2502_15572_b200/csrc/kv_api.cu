// C ABI of the paged key/value cache (the dresd_kv_* calls of include/dresd.h): handle, argument
// validation, workspace.  The kernels are in k10_kv_cache.cu and k11_attend_mma.cu.
#include <cstdarg>
#include <cstdio>
#include <new>

#include "../../include/dresd.h"
#include "internal.h"

using namespace dresd;

namespace {

dresd_status fail(dresd_status st, const char *fmt, ...)
{
    char msg[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(msg, sizeof msg, fmt, ap);
    va_end(ap);
    set_last_error(msg);
    return st;
}
dresd_status fail_cuda(cudaError_t e, const char *what)
{
    return fail(DRESD_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

constexpr uint32_t kKvMagic = 0xD2E5D0C4u;
constexpr int kMaxKvBatch = 65535;
constexpr int kMaxGroup = 64;

bool is_device_ptr(const void *p)
{
    if (!p) return false;
    cudaPointerAttributes at;
    if (cudaPointerGetAttributes(&at, p) != cudaSuccess) {
        cudaGetLastError();
        return false;
    }
    return at.type == cudaMemoryTypeDevice || at.type == cudaMemoryTypeManaged;
}
bool aligned16(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

}  // namespace

struct dresd_kv {
    uint32_t magic;
    int device, sms;
    KvArgs args;                 // arrays and geometry; the batch's part is filled in per call
    float *part;                 // parts of shared items (see kv_plan.cuh)
    unsigned int *tickets;
    cudaStream_t last_stream;
    int last_launches;
};

namespace {

bool valid(const dresd_kv *kv) { return kv && kv->magic == kKvMagic; }

void free_kv(dresd_kv *kv)
{
    cudaFree(kv->part);
    cudaFree(kv->tickets);
    cudaFree(kv->args.status);
    kv->magic = 0;
    delete kv;
}

// Checks the handle and the batch; fills `out` with the cache's arrays and the batch's.
// whole: the call uses start, rows and the layer as well.
dresd_status check_call(dresd_kv *kv, int layer, const dresd_kv_batch *b, bool whole, KvArgs *out)
{
    if (!valid(kv)) return fail(DRESD_ERR_INVALID, "cache handle is NULL or destroyed");
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev != kv->device)
        return fail(DRESD_ERR_INVALID, "the cache belongs to device %d; the current device is %d", kv->device, dev);
    if (!b) return fail(DRESD_ERR_INVALID, "batch is NULL");
    if (layer < 0 || layer >= kv->args.layers) return fail(DRESD_ERR_INVALID, "layer = %d outside 0..%d", layer, kv->args.layers - 1);
    if (b->B < 0) return fail(DRESD_ERR_INVALID, "B = %d is negative", b->B);
    if (b->B > kMaxKvBatch) return fail(DRESD_ERR_UNSUPPORTED, "B = %d exceeds %d", b->B, kMaxKvBatch);
    if (b->table_width < 1) return fail(DRESD_ERR_INVALID, "table_width = %d must be positive", b->table_width);
    if (((long long)b->table_width << kv->args.page_shift) > 2147483647LL)
        return fail(DRESD_ERR_UNSUPPORTED, "table_width = %d reaches beyond 2^31 - 1 positions", b->table_width);
    if (whole && (b->rows < 0 || b->max_chunk < 0 || b->max_chunk > b->rows))
        return fail(DRESD_ERR_INVALID, "rows = %d / max_chunk = %d", b->rows, b->max_chunk);
    *out = kv->args;
    out->layer = layer;
    out->table = b->page_table;
    out->ctx = b->ctx;
    out->start = b->start;
    out->B = b->B;
    out->width = b->table_width;
    out->rows = b->rows;
    if (b->B == 0 || (whole && b->rows == 0)) return DRESD_OK;
    if (!is_device_ptr(b->page_table) || !is_device_ptr(b->ctx) || (whole && !is_device_ptr(b->start)))
        return fail(DRESD_ERR_INVALID, "page_table/ctx/start must be device pointers");
    return DRESD_OK;
}

// Rows of `heads` heads at the given distances: 16-byte loads, and the last one's address within 2^62.
dresd_status check_rows(const char *name, const void *p, long long row, long long head, int heads, int d)
{
    if (!is_device_ptr(p) || !aligned16(p)) return fail(DRESD_ERR_INVALID, "%s must be a 16-byte aligned device pointer", name);
    if (row < 0 || head < 0 || row % 8 != 0 || head % 8 != 0)
        return fail(DRESD_ERR_INVALID, "%s: the distances of rows and heads must be multiples of 8 elements", name);
    if (heads > 1 && head < d) return fail(DRESD_ERR_INVALID, "%s: heads of %d elements overlap at a distance of %lld", name, d, head);
    return DRESD_OK;
}

}  // namespace

extern "C" {

dresd_status dresd_kv_create(void *k_pages, void *v_pages, uint8_t *k_exps, uint8_t *v_exps, int layers,
                             int64_t num_pages, int kv_heads, int page_size, int head_dim, dresd_dtype dtype,
                             dresd_kv **out_kv)
{
    if (!out_kv) return fail(DRESD_ERR_INVALID, "out_kv is NULL");
    *out_kv = nullptr;
    if (!k_pages || !v_pages) return fail(DRESD_ERR_INVALID, "NULL buffer");
    if ((k_exps == nullptr) != (v_exps == nullptr)) return fail(DRESD_ERR_INVALID, "k_exps and v_exps go together");
    if (dtype != DRESD_F32 && dtype != DRESD_F16 && dtype != DRESD_BF16) return fail(DRESD_ERR_INVALID, "unknown dtype %d", (int)dtype);
    if (dtype == DRESD_F32) return fail(DRESD_ERR_UNSUPPORTED, "the cache holds fp16, bf16 or 8-bit rows");
    if (layers < 1 || num_pages < 1 || kv_heads < 1 || page_size < 1 || head_dim < 1)
        return fail(DRESD_ERR_INVALID, "layers = %d, num_pages = %lld, kv_heads = %d, page_size = %d, head_dim = %d", layers,
                    (long long)num_pages, kv_heads, page_size, head_dim);
    if (head_dim != 64 && head_dim != 128) return fail(DRESD_ERR_UNSUPPORTED, "head_dim = %d is not 64 or 128", head_dim);
    if (page_size != 16 && page_size != 32 && page_size != 64 && page_size != 128)
        return fail(DRESD_ERR_UNSUPPORTED, "page_size = %d is not 16, 32, 64 or 128", page_size);
    if (num_pages > 2147483647LL / page_size / kv_heads / layers)
        return fail(DRESD_ERR_UNSUPPORTED, "the cache has more than 2^31 - 1 rows");
    if (!aligned16(k_pages) || !aligned16(v_pages)) return fail(DRESD_ERR_INVALID, "pages not 16-byte aligned");
    if (!is_device_ptr(k_pages) || !is_device_ptr(v_pages) || (k_exps && (!is_device_ptr(k_exps) || !is_device_ptr(v_exps))))
        return fail(DRESD_ERR_INVALID, "k_pages/v_pages/k_exps/v_exps must be device pointers");
    dresd_kv *kv = new (std::nothrow) dresd_kv();
    if (!kv) return fail(DRESD_ERR_ALLOC, "host allocation failed");
    kv->magic = kKvMagic;
    KvArgs &a = kv->args;
    a.k = k_pages;
    a.v = v_pages;
    a.k_exps = k_exps;
    a.v_exps = v_exps;
    a.layers = layers;
    a.heads = kv_heads;
    a.page_shift = page_size == 16 ? 4 : page_size == 32 ? 5 : page_size == 64 ? 6 : 7;
    a.d = head_dim;
    a.dtype = (int)dtype;
    a.num_pages = (int)num_pages;
    cudaError_t e = cudaGetDevice(&kv->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&kv->sms, cudaDevAttrMultiProcessorCount, kv->device);
    if (e != cudaSuccess) {
        free_kv(kv);
        return fail_cuda(e, "device query");
    }
    const size_t tickets = sizeof(unsigned int) * (size_t)attend_max_ctas(kv->sms);
    if (cudaMalloc(&kv->part, sizeof(float) * attend_part_floats(kv->sms, head_dim)) != cudaSuccess ||
        cudaMalloc(&kv->tickets, tickets) != cudaSuccess || cudaMalloc(&a.status, sizeof(int)) != cudaSuccess) {
        cudaGetLastError();
        free_kv(kv);
        return fail(DRESD_ERR_ALLOC, "workspace allocation failed");
    }
    e = cudaMemset(kv->tickets, 0, tickets);
    if (e == cudaSuccess) e = cudaMemset(a.status, 0, sizeof(int));
    if (e == cudaSuccess) e = cudaStreamSynchronize(nullptr);        // other streams may follow at once
    if (e != cudaSuccess) {
        free_kv(kv);
        return fail_cuda(e, "workspace reset");
    }
    *out_kv = kv;
    return DRESD_OK;
}

void dresd_kv_destroy(dresd_kv *kv)
{
    if (valid(kv)) free_kv(kv);
}

dresd_status dresd_kv_append(dresd_kv *kv, int layer, const dresd_kv_batch *batch, const void *k, int64_t k_row,
                             int64_t k_head, const void *v, int64_t v_row, int64_t v_head, void *stream)
{
    KvArgs a;
    dresd_status st = check_call(kv, layer, batch, true, &a);
    if (st != DRESD_OK) return st;
    kv->last_launches = 0;
    if (a.B == 0 || a.rows == 0) return DRESD_OK;
    if ((st = check_rows("k", k, k_row, k_head, a.heads, a.d)) != DRESD_OK) return st;
    if ((st = check_rows("v", v, v_row, v_head, a.heads, a.d)) != DRESD_OK) return st;
    kv->last_stream = static_cast<cudaStream_t>(stream);
    const cudaError_t e = launch_kv_append(a, k, k_row, k_head, v, v_row, v_head, kv->last_stream);
    if (e != cudaSuccess) return fail_cuda(e, "kv_append launch");
    kv->last_launches = 1;
    return DRESD_OK;
}

dresd_status dresd_kv_read(dresd_kv *kv, int layer, const dresd_kv_batch *batch, void *out_k, void *out_v, void *stream)
{
    KvArgs a;
    dresd_status st = check_call(kv, layer, batch, true, &a);
    if (st != DRESD_OK) return st;
    kv->last_launches = 0;
    if (a.B == 0 || a.rows == 0) return DRESD_OK;
    if (!is_device_ptr(out_k) || !is_device_ptr(out_v) || !aligned16(out_k) || !aligned16(out_v))
        return fail(DRESD_ERR_INVALID, "out_k/out_v must be 16-byte aligned device pointers");
    kv->last_stream = static_cast<cudaStream_t>(stream);
    const cudaError_t e = launch_kv_read(a, out_k, out_v, kv->last_stream);
    if (e != cudaSuccess) return fail_cuda(e, "kv_read launch");
    kv->last_launches = 1;
    return DRESD_OK;
}

dresd_status dresd_kv_attend(dresd_kv *kv, int layer, const dresd_kv_batch *batch, const void *q, int64_t q_row,
                             int64_t q_head, int heads, float scale, const uint32_t *mask, int mask_words, void *out,
                             float *out_lse, void *stream)
{
    AttendArgs a{};
    dresd_status st = check_call(kv, layer, batch, true, &a.kv);
    if (st != DRESD_OK) return st;
    if (heads < 1 || heads % a.kv.heads != 0)
        return fail(DRESD_ERR_INVALID, "heads = %d is not a multiple of the cache's %d", heads, a.kv.heads);
    if (heads / a.kv.heads > kMaxGroup)
        return fail(DRESD_ERR_UNSUPPORTED, "%d heads per key/value head exceed %d", heads / a.kv.heads, kMaxGroup);
    if (!(scale - scale == 0.f)) return fail(DRESD_ERR_INVALID, "scale is not finite");
    if (mask && mask_words < 0) return fail(DRESD_ERR_INVALID, "mask_words = %d is negative", mask_words);
    if ((long long)a.kv.rows * (heads / a.kv.heads) > 2147483647LL - 1024)
        return fail(DRESD_ERR_UNSUPPORTED, "rows x heads per key/value head exceed 2^31 - 1025");
    kv->last_launches = 0;
    if (a.kv.B == 0 || a.kv.rows == 0) return DRESD_OK;
    if ((st = check_rows("q", q, q_row, q_head, heads, a.kv.d)) != DRESD_OK) return st;
    if (!is_device_ptr(out) || !aligned16(out) || (out_lse && !is_device_ptr(out_lse)))
        return fail(DRESD_ERR_INVALID, "out must be a 16-byte aligned device pointer, out_lse a device pointer or NULL");
    if (mask && !is_device_ptr(mask)) return fail(DRESD_ERR_INVALID, "mask must be a device pointer");
    a.q = q;
    a.q_row = q_row;
    a.q_head = q_head;
    a.group = heads / a.kv.heads;
    a.scale_log2 = scale * 1.4426950408889634f;
    a.mask = mask;
    a.mask_words = mask_words;
    a.out = out;
    a.lse = out_lse;
    a.part = kv->part;
    a.tickets = kv->tickets;
    a.max_rows = (batch->max_chunk > 0 ? batch->max_chunk : batch->rows) * a.group;
    kv->last_stream = static_cast<cudaStream_t>(stream);
    const cudaError_t e = launch_attend_mma(a, kv->sms, kv->last_stream);
    if (e != cudaSuccess) return fail_cuda(e, "kv_attend launch");
    kv->last_launches = 1;
    return DRESD_OK;
}

dresd_status dresd_kv_keep_draft(dresd_kv *kv, const dresd_kv_batch *batch, const int32_t *best, const int32_t *length,
                                 int n, int L, void *stream)
{
    KvArgs a;
    dresd_status st = check_call(kv, 0, batch, false, &a);
    if (st != DRESD_OK) return st;
    if (n < 1 || L < 1) return fail(DRESD_ERR_INVALID, "bad n/L");
    if (n > DRESD_MAX_TOP_N) return fail(DRESD_ERR_UNSUPPORTED, "n = %d exceeds DRESD_MAX_TOP_N", n);
    if (L > 65536) return fail(DRESD_ERR_UNSUPPORTED, "L = %d exceeds 65536", L);
    kv->last_launches = 0;
    if (a.B == 0) return DRESD_OK;
    if (!is_device_ptr(best) || !is_device_ptr(length)) return fail(DRESD_ERR_INVALID, "best/length must be device pointers");
    kv->last_stream = static_cast<cudaStream_t>(stream);
    const cudaError_t e = launch_kv_keep_draft(a, best, length, n, L, kv->last_stream);
    if (e != cudaSuccess) return fail_cuda(e, "kv_keep_draft launch");
    kv->last_launches = 1;
    return DRESD_OK;
}

dresd_status dresd_kv_status(dresd_kv *kv)
{
    if (!valid(kv)) return fail(DRESD_ERR_INVALID, "cache handle is NULL or destroyed");
    cudaError_t e = cudaStreamSynchronize(kv->last_stream);
    if (e != cudaSuccess) return fail_cuda(e, "stream synchronize");
    int word = 0;
    e = cudaMemcpy(&word, kv->args.status, sizeof(int), cudaMemcpyDeviceToHost);
    if (e != cudaSuccess) return fail_cuda(e, "status read");
    if (word == 0) return DRESD_OK;
    e = cudaMemset(kv->args.status, 0, sizeof(int));
    // a kernel that gave up may have left tickets behind
    if (e == cudaSuccess) e = cudaMemset(kv->tickets, 0, sizeof(unsigned int) * (size_t)attend_max_ctas(kv->sms));
    if (e == cudaSuccess) e = cudaStreamSynchronize(nullptr);
    if (e != cudaSuccess) return fail_cuda(e, "status reset");
    if (word <= -1000) return fail(DRESD_ERR_INTERNAL, "bounds check %d failed inside a kernel", -1000 - word);
    return fail(DRESD_ERR_TIMEOUT, "a device-side wait expired");
}

int dresd_kv_last_launches(const dresd_kv *kv) { return valid(kv) ? kv->last_launches : 0; }

}  // extern "C"
