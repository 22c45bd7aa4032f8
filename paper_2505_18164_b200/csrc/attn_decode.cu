// Attention of one new token per sequence over a paged key/value cache (mdi_attn_decode).
#include "ops_common.cuh"

#include <cuda_fp8.h>

#include <algorithm>

namespace mdi {
namespace {

constexpr int AD_WARPS = 4;

struct AdArgs {
    OpCache c;
    OpRows q, out;
    const int *len;
    int *status;
    int n_head, group, kv_dtype;
    float scale;
};

__device__ __forceinline__ float ad_elem(const AdArgs &a, long long row, int e, int hd) {
    switch (a.kv_dtype) {
        case MDI_KV_F16: return __half2float(((const __half *)a.c.pool)[row * hd + e]);
        case MDI_KV_BF16: return __bfloat162float(((const __nv_bfloat16 *)a.c.pool)[row * hd + e]);
        case MDI_KV_I8: return (float)((const signed char *)a.c.pool)[row * hd + e] * a.c.scale[row];
        default: return (float)((const __nv_fp8_e4m3 *)a.c.pool)[row * hd + e] * a.c.scale[row];
    }
}

// grid (n_head, n_seq): one block per head and sequence, a warp per cached row at a time, online softmax.
template <typename RT>
__global__ void __launch_bounds__(AD_WARPS * 32) k_attn_decode_op(const AdArgs a) {
    __shared__ float sm_m[AD_WARPS], sm_l[AD_WARPS], sm_o[AD_WARPS][128];
    const int h = blockIdx.x, i = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, hd = a.c.head_dim;
    const int slot = op_slot(a.c, i);
    long long len = a.len[i];
    if (slot < 0 || len < 0 || len > a.c.capacity) {
        if (tid == 0) op_status(a.status, MDI_STATUS_RANGE);
        len = slot < 0 || len < 0 ? 0 : a.c.capacity;
    }
    const RT *q = (const RT *)a.q.data + i * a.q.row_stride + h * a.q.head_stride;
    float qv[4], o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;
#pragma unroll
    for (int u = 0; u < 4; ++u) qv[u] = lane + 32 * u < hd ? (float)q[lane + 32 * u] * a.scale : 0.f;
    for (long long t = warp; t < len; t += AD_WARPS) {
        const int p = a.c.table[(long long)slot * a.c.table_stride + (t >> a.c.page_shift)];
        if ((unsigned)p >= (unsigned)a.c.n_pages) {
            if (lane == 0) op_status(a.status, MDI_STATUS_PAGE);
            continue;
        }
        const long long kr = ((((long long)p * 2) * a.c.n_kv_head + h / a.group) << a.c.page_shift) + (t & ((1 << a.c.page_shift) - 1));
        const long long vr = kr + ((long long)a.c.n_kv_head << a.c.page_shift);
        float s = 0.f;
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (lane + 32 * u < hd) s = fmaf(qv[u], ad_elem(a, kr, lane + 32 * u, hd), s);
#pragma unroll
        for (int w = 16; w > 0; w >>= 1) s += __shfl_xor_sync(0xffffffffu, s, w);
        const float mn = fmaxf(m, s), ref = mn == -INFINITY ? 0.f : mn, corr = expf(m - ref), pr = expf(s - ref);
        l = l * corr + pr;
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (lane + 32 * u < hd) o[u] = o[u] * corr + pr * ad_elem(a, vr, lane + 32 * u, hd);
        m = mn;
    }
    if (lane == 0) { sm_m[warp] = m; sm_l[warp] = l; }
#pragma unroll
    for (int u = 0; u < 4; ++u) sm_o[warp][lane + 32 * u] = o[u];
    __syncthreads();
    if (tid < hd) {
        float M = -INFINITY, L = 0.f, O = 0.f;
        for (int w = 0; w < AD_WARPS; ++w) M = fmaxf(M, sm_m[w]);
        if (M == -INFINITY) M = 0.f;
        for (int w = 0; w < AD_WARPS; ++w) { const float f = expf(sm_m[w] - M); L += sm_l[w] * f; O += sm_o[w][tid] * f; }
        RT *out = (RT *)a.out.data + i * a.out.row_stride + h * a.out.head_stride;
        out[tid] = (RT)(len == 0 ? 0.f : O / L);
    }
}

int ad_check(const char *who, const mdi_kv_cache *cache, int n_seq, int n_head, int max_len) {
    const int rc = op_check_cache(who, cache);
    if (rc != MDI_OK) return rc;
    if (n_seq < 0 || n_seq > 65535) return op_fail(MDI_ERR_ARG, "%s: n_seq must be in 0..65535", who);
    if (max_len < 0) return op_fail(MDI_ERR_ARG, "%s: negative max_len", who);
    if (n_head < 1 || n_head % cache->n_kv_head || n_head / cache->n_kv_head > 64)
        return op_fail(MDI_ERR_SHAPE, "%s: n_head must be a multiple of n_kv_head, at most 64 heads each", who);
    return MDI_OK;
}

} // namespace
} // namespace mdi

using namespace mdi;

extern "C" int64_t mdi_attn_decode_workspace(const mdi_kv_cache *cache, int n_seq, int n_head, int max_len) {
    const int rc = ad_check("mdi_attn_decode_workspace", cache, n_seq, n_head, max_len);
    return rc != MDI_OK ? rc : 0;
}

extern "C" int mdi_attn_decode(const mdi_kv_cache *cache, int n_seq, const int32_t *slot_dev, const int32_t *len_dev, int max_len, int n_head,
                               const mdi_rows *q, const mdi_rows *out, float scale, void *workspace_dev, int64_t workspace_bytes,
                               int32_t *status_dev, void *stream) {
    const char *who = "mdi_attn_decode";
    int rc = ad_check(who, cache, n_seq, n_head, max_len);
    if (rc != MDI_OK) return rc;
    if (!slot_dev && n_seq > cache->n_slots) return op_fail(MDI_ERR_ARG, "%s: %d sequences, but the page table has %d slots", who, n_seq, cache->n_slots);
    if (!(scale > 0.f) || scale > 3e38f) return op_fail(MDI_ERR_ARG, "%s: scale must be positive and finite", who);
    if ((rc = op_check_rows(who, "q", q, n_seq, n_head)) != MDI_OK) return rc;
    if ((rc = op_check_rows(who, "out", out, n_seq, n_head)) != MDI_OK) return rc;
    if (q->dtype != out->dtype) return op_fail(MDI_ERR_ARG, "%s: q and out differ in dtype", who);
    if ((rc = op_check_ptrs(who, {{"pool_dev", cache->pool_dev, false}, {"scale_dev", cache->scale_dev, !op_scaled(cache)}, {"page_table_dev", cache->page_table_dev, false},
                                  {"q", q->data_dev, n_seq == 0}, {"out", out->data_dev, n_seq == 0}, {"slot_dev", slot_dev, true},
                                  {"len_dev", len_dev, false}, {"workspace_dev", workspace_dev, true}, {"status_dev", status_dev, true}})) != MDI_OK)
        return rc;
    if (n_seq == 0) return MDI_OK;
    (void)workspace_dev; (void)workspace_bytes;
    AdArgs a{};
    a.c = op_cache(cache, slot_dev);
    a.q = op_rows(q); a.out = op_rows(out);
    a.len = len_dev; a.status = status_dev;
    a.n_head = n_head; a.group = n_head / cache->n_kv_head; a.kv_dtype = cache->dtype; a.scale = scale;
    OP_ROW_DISPATCH(q->dtype, (k_attn_decode_op<RT><<<dim3(n_head, n_seq), AD_WARPS * 32, 0, (cudaStream_t)stream>>>(a)));
    return op_cuda(who, cudaGetLastError());
}
