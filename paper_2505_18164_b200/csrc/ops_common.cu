// Checks of the operators' arguments (ops_common.cuh).
#include "ops_common.cuh"

#include <cstdarg>
#include <cstdio>

namespace mdi {

int op_fail(int code, const char *fmt, ...) {
    char buf[384];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    mdi_internal_set_error(buf);
    return code;
}

int op_cuda(const char *who, cudaError_t e) {
    return e == cudaSuccess ? MDI_OK : op_fail(MDI_ERR_CUDA, "%s: %s", who, cudaGetErrorString(e));
}

int op_check_ptrs(const char *who, std::initializer_list<OpPtr> ptrs) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    for (const OpPtr &x : ptrs) {
        if (!x.p) {
            if (x.optional) continue;
            return op_fail(MDI_ERR_ARG, "%s: %s is null", who, x.name);
        }
        cudaPointerAttributes a;
        if (e == cudaSuccess) e = cudaPointerGetAttributes(&a, x.p);
        if (e != cudaSuccess) {
            cudaGetLastError();
            return op_fail(MDI_ERR_CUDA, "%s: %s: %s", who, x.name, cudaGetErrorString(e));
        }
        if (a.type != cudaMemoryTypeDevice && a.type != cudaMemoryTypeManaged) return op_fail(MDI_ERR_ARG, "%s: %s is not device memory", who, x.name);
        if (a.type == cudaMemoryTypeDevice && a.device != dev)
            return op_fail(MDI_ERR_ARG, "%s: %s is memory of device %d, the current device is %d", who, x.name, a.device, dev);
    }
    return MDI_OK;
}

int op_check_rows(const char *who, const char *name, const mdi_rows *r, int rows, int heads, bool written) {
    if (!r) return op_fail(MDI_ERR_ARG, "%s: %s is null", who, name);
    if (r->dtype != MDI_DTYPE_F32 && r->dtype != MDI_DTYPE_BF16 && r->dtype != MDI_DTYPE_F16) return op_fail(MDI_ERR_ARG, "%s: %s: unknown dtype", who, name);
    const int64_t unit = r->dtype == MDI_DTYPE_F32 ? 4 : 8; // elements in 16 bytes
    if (((uintptr_t)r->data_dev & 15) || (rows > 1 && r->row_stride % unit) || (heads > 1 && r->head_stride % unit))
        return op_fail(MDI_ERR_SHAPE, "%s: %s: the data and its strides must be multiples of 16 bytes", who, name);
    if (written && ((rows > 1 && r->row_stride == 0) || (heads > 1 && r->head_stride == 0))) return op_fail(MDI_ERR_SHAPE, "%s: %s: a stride of an output is zero", who, name);
    if ((rows > 1 && r->row_stride < 0) || (heads > 1 && r->head_stride < 0)) return op_fail(MDI_ERR_SHAPE, "%s: %s: negative stride", who, name);
    return MDI_OK;
}

int op_check_cache(const char *who, const mdi_kv_cache *c) {
    if (!c) return op_fail(MDI_ERR_ARG, "%s: cache is null", who);
    if (c->dtype != MDI_KV_F16 && c->dtype != MDI_KV_BF16 && c->dtype != MDI_KV_I8 && c->dtype != MDI_KV_E4M3)
        return op_fail(MDI_ERR_ARG, "%s: the cache's dtype must be MDI_KV_F16, _BF16, _I8 or _E4M3", who);
    if (c->n_pages < 1 || c->n_slots < 1 || c->pages_per_seq < 1 || c->page_table_stride < c->pages_per_seq)
        return op_fail(MDI_ERR_ARG, "%s: the cache needs pages, slots and a page table with page_table_stride >= pages_per_seq", who);
    if (c->head_dim != 16 && c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128)
        return op_fail(MDI_ERR_SHAPE, "%s: head_dim must be 16, 32, 64 or 128", who);
    if (c->page_tokens < 16 || c->page_tokens > (1 << 20) || (c->page_tokens & (c->page_tokens - 1)))
        return op_fail(MDI_ERR_SHAPE, "%s: page_tokens must be a power of two >= 16", who);
    if (c->n_kv_head < 1 || c->n_kv_head > 1024) return op_fail(MDI_ERR_SHAPE, "%s: n_kv_head must be in 1..1024", who);
    if (((uintptr_t)c->pool_dev & 15) || (op_scaled(c) && ((uintptr_t)c->scale_dev & 15))) return op_fail(MDI_ERR_SHAPE, "%s: pool and scales must be 16-byte aligned", who);
    return MDI_OK;
}

OpCache op_cache(const mdi_kv_cache *c, const int32_t *slot_dev) {
    OpCache d{};
    d.pool = (unsigned char *)c->pool_dev;
    d.scale = c->scale_dev;
    d.table = c->page_table_dev;
    d.slot = slot_dev;
    d.table_stride = c->page_table_stride;
    d.n_pages = c->n_pages; d.n_slots = c->n_slots; d.pages_per_seq = c->pages_per_seq;
    d.n_kv_head = c->n_kv_head; d.head_dim = c->head_dim;
    while ((1 << d.page_shift) < c->page_tokens) ++d.page_shift;
    d.capacity = (long long)c->pages_per_seq << d.page_shift;
    return d;
}

} // namespace mdi
