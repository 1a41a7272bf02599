// C ABI of the paged key/value cache (the dresd_kv_* calls of include/dresd.h): handle, argument
// validation, tensor maps, workspace.  The kernels are in k10_kv_cache.cu, k11_attend_mma.cu,
// k12_attend_umma.cu and k14_kv_pages.cu.
#include <cstring>
#include <new>

#include "api_util.h"

using namespace dresd;

namespace {

constexpr uint32_t kKvMagic = 0xD2E5D0C4u;
constexpr int kMaxKvBatch = 65535;
constexpr int kMaxGroup = 64;

bool aligned16(const void *p) { return aligned(p, 16); }

}  // namespace

struct dresd_kv {
    uint32_t magic;
    int device, sms;
    CUtensorMap k_map, v_map;    // over the cache's rows, boxes of a page (tcgen05 kernel)
    CUtensorMap k16_map, v16_map;    // boxes of 16 rows (mma.sync kernel)
    KvArgs args;                 // arrays and geometry; the batch's part is filled in per call
    float *part;                 // parts of shared items (see kv_plan.cuh)
    unsigned int *tickets;
    PageArgs pages;              // refs is null until dresd_kv_attach_pages()
    int opt_path, opt_wait_ms, opt_lose_stage;
    cudaStream_t last_stream;
    int last_launches;
};

namespace {

bool valid(const dresd_kv *kv) { return kv && kv->magic == kKvMagic; }

void free_kv(dresd_kv *kv)
{
    cudaFree(kv->part);
    cudaFree(kv->tickets);
    cudaFree(kv->pages.last);     // all of the pages' workspace
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
    if (((long long)b->table_width << kv->args.page_shift) > 2147483647LL - 4096)
        return fail(DRESD_ERR_UNSUPPORTED, "table_width = %d reaches beyond 2^31 - 4097 positions", b->table_width);
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
    if (!is_device_ptr(b->page_table, dev) || !is_device_ptr(b->ctx, dev) || (whole && !is_device_ptr(b->start, dev)))
        return fail(DRESD_ERR_INVALID, "page_table/ctx/start must be pointers of the cache's device");
    return DRESD_OK;
}

// The same for a call that counts pages and writes the table.
dresd_status check_pages(dresd_kv *kv, const dresd_kv_batch *b, bool whole, KvArgs *out)
{
    const dresd_status st = check_call(kv, 0, b, whole, out);
    if (st != DRESD_OK) return st;
    if (!kv->pages.refs) return fail(DRESD_ERR_INVALID, "the cache has no page counts: dresd_kv_attach_pages() comes first");
    if (!aligned(b->page_table, 4) || !aligned(b->ctx, 4) || (whole && !aligned(b->start, 4)))
        return fail(DRESD_ERR_INVALID, "page_table/ctx/start must be 4-byte aligned");
    return DRESD_OK;
}

// Rows of `heads` heads at the given distances: 16-byte loads.
dresd_status check_rows(const dresd_kv *kv, const char *name, const void *p, int rows, long long row, long long head, int heads)
{
    const int d = kv->args.d;
    if (!is_device_ptr(p, kv->device) || !aligned16(p))
        return fail(DRESD_ERR_INVALID, "%s must be a 16-byte aligned pointer of the cache's device", name);
    if (row < 0 || head < 0 || row % 8 != 0 || head % 8 != 0)
        return fail(DRESD_ERR_INVALID, "%s: the distances of rows and heads must be multiples of 8 elements", name);
    if ((heads > 1 && (head < d || head >= 1LL << 38)) || (rows > 1 && (row < d || row >= 1LL << 38)))
        return fail(DRESD_ERR_INVALID, "%s: distances of %lld (rows) and %lld (heads) elements for heads of %d", name, row, head, d);
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
    if (k_exps && (!aligned16(k_exps) || !aligned16(v_exps))) return fail(DRESD_ERR_INVALID, "exponents not 16-byte aligned");
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess) cudaGetLastError();       // then no pointer is one of it
    if (!is_device_ptr(k_pages, dev) || !is_device_ptr(v_pages, dev) || (k_exps && (!is_device_ptr(k_exps, dev) || !is_device_ptr(v_exps, dev))))
        return fail(DRESD_ERR_INVALID, "k_pages/v_pages/k_exps/v_exps must be pointers of the current device");
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
    kv->device = dev;
    cudaError_t e = cudaDeviceGetAttribute(&kv->sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) {
        free_kv(kv);
        return fail_cuda(e, "device query");
    }
    const size_t tickets = sizeof(unsigned int) * attend_mma_workers(kv->sms);
    const size_t few = attend_mma_part_floats(kv->sms, head_dim), many = attend_umma_part_floats(kv->sms, head_dim);
    const cuuint64_t dims[2] = {(cuuint64_t)head_dim, (cuuint64_t)layers * num_pages * kv_heads * page_size};
    const cuuint64_t strides[1] = {(cuuint64_t)head_dim * (k_exps ? 1 : 2)};
    const cuuint32_t box[2] = {(cuuint32_t)(k_exps ? head_dim : 64), (cuuint32_t)page_size};
    const cuuint32_t box16[2] = {box[0], 16};
    const int held = k_exps ? kE4M3 : a.dtype;
    const CUtensorMapSwizzle none = k_exps ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B;
    const CUtensorMapSwizzle row = k_exps && head_dim == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B;
    if (!encode(&kv->k_map, k_pages, held, 2, dims, strides, box, none) || !encode(&kv->v_map, v_pages, held, 2, dims, strides, box, none) ||
        !encode(&kv->k16_map, k_pages, held, 2, dims, strides, box16, row) || !encode(&kv->v16_map, v_pages, held, 2, dims, strides, box16, row)) {
        free_kv(kv);
        return fail(DRESD_ERR_CUDA, "cuTensorMapEncodeTiled failed");
    }
    if (cudaMalloc(&kv->part, sizeof(float) * (few > many ? few : many)) != cudaSuccess ||
        cudaMalloc(&kv->tickets, tickets) != cudaSuccess || cudaMalloc(&a.status, sizeof(int)) != cudaSuccess) {
        cudaGetLastError();
        free_kv(kv);
        return fail(DRESD_ERR_ALLOC, "workspace allocation failed");
    }
    // On a stream of its own: any stream may follow at once, and what others have queued is not waited for.
    cudaStream_t own = nullptr;
    e = cudaStreamCreateWithFlags(&own, cudaStreamNonBlocking);
    if (e == cudaSuccess) e = cudaMemsetAsync(kv->tickets, 0, tickets, own);
    if (e == cudaSuccess) e = cudaMemsetAsync(a.status, 0, sizeof(int), own);
    if (e == cudaSuccess) e = cudaStreamSynchronize(own);
    if (own) cudaStreamDestroy(own);
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
    if ((st = check_rows(kv, "k", k, a.rows, k_row, k_head, a.heads)) != DRESD_OK) return st;
    if ((st = check_rows(kv, "v", v, a.rows, v_row, v_head, a.heads)) != DRESD_OK) return st;
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
    if (!is_device_ptr(out_k, kv->device) || !is_device_ptr(out_v, kv->device) || !aligned16(out_k) || !aligned16(out_v))
        return fail(DRESD_ERR_INVALID, "out_k/out_v must be 16-byte aligned pointers of the cache's device");
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
    if ((st = check_rows(kv, "q", q, a.kv.rows, q_row, q_head, heads)) != DRESD_OK) return st;
    if (!is_device_ptr(out, kv->device) || !aligned16(out) || (out_lse && !is_device_ptr(out_lse, kv->device)))
        return fail(DRESD_ERR_INVALID, "out must be a 16-byte aligned pointer of the cache's device, out_lse one of it or NULL");
    if (mask && !is_device_ptr(mask, kv->device)) return fail(DRESD_ERR_INVALID, "mask must be a pointer of the cache's device");
    a.q = q;
    a.q_row = q_row;
    a.q_head = q_head;
    a.group = heads / a.kv.heads;
    a.by_group = FastDiv(a.group);
    a.scale_log2 = scale * 1.4426950408889634f;
    a.mask = mask;
    a.mask_words = mask_words;
    a.out = out;
    a.lse = out_lse;
    a.part = kv->part;
    a.tickets = kv->tickets;
    a.max_chunk = batch->max_chunk > 0 ? batch->max_chunk : batch->rows;
    a.wait_cycles = (long long)kv->opt_wait_ms * 2000000LL;        // ~2 GHz
    a.lose_stage = kv->opt_lose_stage;
    kv->last_stream = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    // Up to 16 rows per key/value head the registers of mma.sync hold them: 16 sequences of 8000, 8 heads of 128, 16 rows 88 us
    // with that kernel and 93 with the other (8 bits: 90 and 128), 32 rows 167 and 94 (171 and 131); one of 2000, 32
    // heads, 16 rows 14.5 and 20.9, 17 rows 19.5 and 21.1.  The other kernel masks before it scales, which needs a positive scale.
    const bool many = kv->opt_path == 0 ? (long long)a.max_chunk * a.group > 16 : kv->opt_path == 2;
    if (many && scale > 0.f) {
        CUtensorMap q_map;
        const cuuint64_t dims[3] = {(cuuint64_t)a.kv.d, (cuuint64_t)heads, (cuuint64_t)a.kv.rows};
        // the distance of a dimension with one entry is never used, but has to be a valid one
        const cuuint64_t strides[2] = {heads > 1 ? (cuuint64_t)q_head * 2 : (cuuint64_t)a.kv.d * 2,
                                       a.kv.rows > 1 ? (cuuint64_t)q_row * 2 : (cuuint64_t)heads * a.kv.d * 2};
        const cuuint32_t box[3] = {64, (cuuint32_t)a.group, (cuuint32_t)(128 / a.group)};
        if (!encode(&q_map, q, a.kv.dtype, 3, dims, strides, box)) return fail(DRESD_ERR_CUDA, "cuTensorMapEncodeTiled failed for q");
        e = launch_attend_umma(q_map, kv->k_map, kv->v_map, a, kv->sms, kv->last_stream);
    } else {
        e = launch_attend_mma(kv->k16_map, kv->v16_map, a, kv->sms, kv->last_stream);
    }
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
    if (!is_device_ptr(best, kv->device) || !is_device_ptr(length, kv->device))
        return fail(DRESD_ERR_INVALID, "best/length must be pointers of the cache's device");
    kv->last_stream = static_cast<cudaStream_t>(stream);
    const cudaError_t e = launch_kv_keep_draft(a, best, length, n, L, kv->last_stream);
    if (e != cudaSuccess) return fail_cuda(e, "kv_keep_draft launch");
    kv->last_launches = 1;
    return DRESD_OK;
}

dresd_status dresd_kv_attach_pages(dresd_kv *kv, int32_t *refs)
{
    if (!valid(kv)) return fail(DRESD_ERR_INVALID, "cache handle is NULL or destroyed");
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev != kv->device)
        return fail(DRESD_ERR_INVALID, "the cache belongs to device %d; the current device is %d", kv->device, dev);
    if (!is_word_ptr(refs, dev))
        return fail(DRESD_ERR_INVALID, "refs must be an aligned pointer of the cache's device");
    if (!kv->pages.last) {
        const size_t n = (size_t)kv->args.num_pages, words = 7 * n + kMaxKvBatch + kPageCounts;
        PageArgs w{};
        if (cudaMalloc(&w.last, 4 * words) != cudaSuccess) {
            cudaGetLastError();
            return fail(DRESD_ERR_ALLOC, "workspace allocation failed");
        }
        w.holders = reinterpret_cast<int32_t *>(w.last + n);
        w.map = w.holders + n;
        w.list = w.map + n;
        w.from = w.list + n;
        w.to = w.from + n;
        w.row_first = w.to + n;
        w.counts = w.row_first + kMaxKvBatch;
        // on a stream of its own, as in dresd_kv_create()
        cudaStream_t own = nullptr;
        cudaError_t e = cudaStreamCreateWithFlags(&own, cudaStreamNonBlocking);
        if (e == cudaSuccess) e = cudaMemsetAsync(w.last, 0, 4 * words, own);
        if (e == cudaSuccess) e = cudaStreamSynchronize(own);
        if (own) cudaStreamDestroy(own);
        if (e != cudaSuccess) {
            cudaFree(w.last);
            return fail_cuda(e, "workspace reset");
        }
        kv->pages = w;
    }
    kv->pages.refs = refs;
    return DRESD_OK;
}

dresd_status dresd_kv_fork(dresd_kv *kv, const dresd_kv_batch *batch, int32_t *ctx, const int32_t *parent, void *stream)
{
    KvArgs a;
    dresd_status st = check_pages(kv, batch, false, &a);
    if (st != DRESD_OK) return st;
    kv->last_launches = 0;
    if (a.B == 0) return DRESD_OK;
    if (ctx != a.ctx) return fail(DRESD_ERR_INVALID, "ctx must be the batch's");
    if (!is_word_ptr(parent, kv->device)) return fail(DRESD_ERR_INVALID, "parent must be an aligned pointer of the cache's device");
    kv->last_stream = static_cast<cudaStream_t>(stream);
    const cudaError_t e = launch_kv_fork(a, kv->pages.refs, const_cast<int32_t *>(a.table), ctx, parent, kv->last_stream);
    if (e != cudaSuccess) return fail_cuda(e, "kv_fork launch");
    kv->last_launches = 1;
    return DRESD_OK;
}

dresd_status dresd_kv_reserve(dresd_kv *kv, const dresd_kv_batch *batch, int32_t *out_missing, void *stream)
{
    KvArgs a;
    dresd_status st = check_pages(kv, batch, true, &a);
    if (st != DRESD_OK) return st;
    kv->last_launches = 0;
    if (!is_word_ptr(out_missing, kv->device)) return fail(DRESD_ERR_INVALID, "out_missing must be an aligned pointer of the cache's device");
    kv->last_stream = static_cast<cudaStream_t>(stream);
    if (a.B == 0 || a.rows == 0) {
        const cudaError_t e = cudaMemsetAsync(out_missing, 0, sizeof(int32_t), kv->last_stream);
        return e == cudaSuccess ? DRESD_OK : fail_cuda(e, "kv_reserve");
    }
    const cudaError_t e = launch_kv_reserve(a, kv->pages, const_cast<int32_t *>(a.table), out_missing, kv->sms, kv->last_stream);
    if (e != cudaSuccess) return fail_cuda(e, "kv_reserve launch");
    kv->last_launches = 2;
    return DRESD_OK;
}

dresd_status dresd_kv_release(dresd_kv *kv, const dresd_kv_batch *batch, const int32_t *keep, void *stream)
{
    KvArgs a;
    dresd_status st = check_pages(kv, batch, false, &a);
    if (st != DRESD_OK) return st;
    kv->last_launches = 0;
    if (a.B == 0) return DRESD_OK;
    if (!is_word_ptr(keep, kv->device)) return fail(DRESD_ERR_INVALID, "keep must be an aligned pointer of the cache's device");
    kv->last_stream = static_cast<cudaStream_t>(stream);
    const cudaError_t e = launch_kv_release(a, kv->pages.refs, const_cast<int32_t *>(a.table), keep, kv->last_stream);
    if (e != cudaSuccess) return fail_cuda(e, "kv_release launch");
    kv->last_launches = 1;
    return DRESD_OK;
}

dresd_status dresd_kv_compact(dresd_kv *kv, const dresd_kv_batch *batch, int32_t *out_used, void *stream)
{
    KvArgs a;
    dresd_status st = check_pages(kv, batch, false, &a);
    if (st != DRESD_OK) return st;
    kv->last_launches = 0;
    if (!is_word_ptr(out_used, kv->device)) return fail(DRESD_ERR_INVALID, "out_used must be an aligned pointer of the cache's device");
    kv->last_stream = static_cast<cudaStream_t>(stream);
    const cudaError_t e = launch_kv_compact(a, kv->pages, const_cast<int32_t *>(a.table), out_used, kv->sms, kv->last_stream);
    if (e != cudaSuccess) return fail_cuda(e, "kv_compact launch");
    kv->last_launches = 2;
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
    if (e == cudaSuccess) e = cudaMemset(kv->tickets, 0, sizeof(unsigned int) * attend_mma_workers(kv->sms));
    if (e == cudaSuccess) e = cudaStreamSynchronize(nullptr);
    if (e != cudaSuccess) return fail_cuda(e, "status reset");
    if (word <= -1000) return fail(DRESD_ERR_INTERNAL, "debug build: bounds check %d failed (an index or ring slot out of range)", -1000 - word);
    return fail(DRESD_ERR_TIMEOUT, "a device-side wait expired");
}

dresd_status dresd_kv_set_option(dresd_kv *kv, const char *name, int value)
{
    if (!valid(kv) || !name) return fail(DRESD_ERR_INVALID, "cache handle or option name is NULL");
    if (strcmp(name, "attend_path") == 0) {
        if (value < 0 || value > 2) return fail(DRESD_ERR_INVALID, "attend_path = %d outside 0..2", value);
        kv->opt_path = value;
        return DRESD_OK;
    }
    if (strcmp(name, "wait_ms") == 0) {
        if (value < 0 || value > 60000) return fail(DRESD_ERR_INVALID, "wait_ms = %d outside 0..60000", value);
        kv->opt_wait_ms = value;
        return DRESD_OK;
    }
    if (strcmp(name, "debug_lose_stage") == 0) {
        if (value < 0) return fail(DRESD_ERR_INVALID, "debug_lose_stage = %d is negative", value);
        kv->opt_lose_stage = value;
        return DRESD_OK;
    }
    return fail(DRESD_ERR_INVALID, "unknown option '%s'", name);
}

dresd_status dresd_kv_debug_selftest(dresd_kv *kv, void *stream)
{
    if (!valid(kv)) return fail(DRESD_ERR_INVALID, "cache handle is NULL or destroyed");
#ifdef DRESD_DEBUG_BOUNDS
    kv->last_stream = static_cast<cudaStream_t>(stream);
    const cudaError_t e = launch_debug_selftest(kv->args.status, kv->last_stream);
    return e == cudaSuccess ? DRESD_OK : fail_cuda(e, "selftest launch");
#else
    (void)stream;
    return fail(DRESD_ERR_UNSUPPORTED, "this is the release build: no bounds checks are compiled in");
#endif
}

int dresd_kv_last_launches(const dresd_kv *kv) { return valid(kv) ? kv->last_launches : 0; }

}  // extern "C"
