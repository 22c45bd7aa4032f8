// Causal attention over packed sequences (mdi_attn_prompt).
#include "ops_common.cuh"

#include <algorithm>

namespace mdi {
namespace {

constexpr int AP_WARPS = 4;

struct ApArgs {
    OpRows q, k, v, out;
    const int *q_start, *k_start;
    int *status;
    int n_seq, n_q, n_k, group, hd;
    float scale;
};

// grid (n_head, query rows): a warp per key row at a time, online softmax.
template <typename RT>
__global__ void __launch_bounds__(AP_WARPS * 32) k_attn_prompt_rows(const ApArgs a) {
    __shared__ float sm_m[AP_WARPS], sm_l[AP_WARPS], sm_o[AP_WARPS][128];
    const int h = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, hd = a.hd;
    for (int row = blockIdx.y; row < a.n_q; row += gridDim.y) {
        if (row >= a.q_start[a.n_seq]) return;
        const int i = op_find(a.q_start, a.n_seq, row);
        const int q0 = a.q_start[i], q1 = a.q_start[i + 1], k0 = a.k_start[i], k1 = a.k_start[i + 1];
        if (i == 0 && row < q0) continue;
        if (row < q0 || row >= q1 || q1 > a.n_q || k0 < 0 || k1 < k0 || k1 > a.n_k) {
            if (tid == 0) op_status(a.status, MDI_STATUS_RANGE);
            continue;
        }
        const int seen = max(0, k1 - k0 - (q1 - q0) + (row - q0) + 1); // keys this row sees
        const RT *q = (const RT *)a.q.data + row * a.q.row_stride + h * a.q.head_stride;
        float qv[4], o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;
#pragma unroll
        for (int u = 0; u < 4; ++u) qv[u] = lane + 32 * u < hd ? (float)q[lane + 32 * u] * a.scale : 0.f;
        for (int j = warp; j < seen; j += AP_WARPS) {
            const RT *k = (const RT *)a.k.data + (k0 + j) * a.k.row_stride + h / a.group * a.k.head_stride;
            const RT *v = (const RT *)a.v.data + (k0 + j) * a.v.row_stride + h / a.group * a.v.head_stride;
            float s = 0.f;
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (lane + 32 * u < hd) s = fmaf(qv[u], (float)k[lane + 32 * u], s);
#pragma unroll
            for (int w = 16; w > 0; w >>= 1) s += __shfl_xor_sync(0xffffffffu, s, w);
            const float mn = fmaxf(m, s), ref = mn == -INFINITY ? 0.f : mn, corr = expf(m - ref), pr = expf(s - ref);
            l = l * corr + pr;
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (lane + 32 * u < hd) o[u] = o[u] * corr + pr * (float)v[lane + 32 * u];
            m = mn;
        }
        __syncthreads();
        if (lane == 0) { sm_m[warp] = m; sm_l[warp] = l; }
#pragma unroll
        for (int u = 0; u < 4; ++u) sm_o[warp][lane + 32 * u] = o[u];
        __syncthreads();
        if (tid < hd) {
            float M = -INFINITY, L = 0.f, O = 0.f;
            for (int w = 0; w < AP_WARPS; ++w) M = fmaxf(M, sm_m[w]);
            if (M == -INFINITY) M = 0.f;
            for (int w = 0; w < AP_WARPS; ++w) { const float f = expf(sm_m[w] - M); L += sm_l[w] * f; O += sm_o[w][tid] * f; }
            RT *out = (RT *)a.out.data + row * a.out.row_stride + h * a.out.head_stride;
            out[tid] = (RT)(seen == 0 ? 0.f : O / L);
        }
    }
}

} // namespace
} // namespace mdi

using namespace mdi;

extern "C" int mdi_attn_prompt(int n_seq, const int32_t *q_start_dev, const int32_t *k_start_dev, int n_q_rows, int n_k_rows, int n_head, int n_kv_head,
                               int head_dim, const mdi_rows *q, const mdi_rows *k, const mdi_rows *v, const mdi_rows *out, float scale,
                               int32_t *status_dev, void *stream) {
    const char *who = "mdi_attn_prompt";
    int rc;
    if (n_seq < 0 || n_q_rows < 0 || n_k_rows < 0) return op_fail(MDI_ERR_ARG, "%s: negative n_seq, n_q_rows or n_k_rows", who);
    if (head_dim != 16 && head_dim != 32 && head_dim != 64 && head_dim != 128) return op_fail(MDI_ERR_SHAPE, "%s: head_dim must be 16, 32, 64 or 128", who);
    if (n_kv_head < 1 || n_head < 1 || n_head % n_kv_head || n_head > 65535) return op_fail(MDI_ERR_SHAPE, "%s: n_head must be a multiple of n_kv_head", who);
    if (!(scale > 0.f) || scale > 3e38f) return op_fail(MDI_ERR_ARG, "%s: scale must be positive and finite", who);
    if ((rc = op_check_rows(who, "q", q, n_q_rows, n_head)) != MDI_OK) return rc;
    if ((rc = op_check_rows(who, "k", k, n_k_rows, n_kv_head)) != MDI_OK) return rc;
    if ((rc = op_check_rows(who, "v", v, n_k_rows, n_kv_head)) != MDI_OK) return rc;
    if ((rc = op_check_rows(who, "out", out, n_q_rows, n_head)) != MDI_OK) return rc;
    if ((q->dtype != MDI_DTYPE_F16 && q->dtype != MDI_DTYPE_BF16) || k->dtype != q->dtype || v->dtype != q->dtype || out->dtype != q->dtype)
        return op_fail(MDI_ERR_ARG, "%s: q, k, v and out must share one dtype, F16 or BF16", who);
    if ((rc = op_check_ptrs(who, {{"q", q->data_dev, n_q_rows == 0}, {"k", k->data_dev, n_k_rows == 0}, {"v", v->data_dev, n_k_rows == 0}, {"out", out->data_dev, n_q_rows == 0},
                                  {"q_start_dev", q_start_dev, false}, {"k_start_dev", k_start_dev, false}, {"status_dev", status_dev, true}})) != MDI_OK)
        return rc;
    if (n_seq == 0 || n_q_rows == 0) return MDI_OK;
    ApArgs a{};
    a.q = op_rows(q); a.k = op_rows(k); a.v = op_rows(v); a.out = op_rows(out);
    a.q_start = q_start_dev; a.k_start = k_start_dev; a.status = status_dev;
    a.n_seq = n_seq; a.n_q = n_q_rows; a.n_k = n_k_rows; a.group = n_head / n_kv_head; a.hd = head_dim; a.scale = scale;
    const dim3 grid(n_head, std::min(n_q_rows, 65535));
    if (q->dtype == MDI_DTYPE_F16) k_attn_prompt_rows<__half><<<grid, AP_WARPS * 32, 0, (cudaStream_t)stream>>>(a);
    else k_attn_prompt_rows<__nv_bfloat16><<<grid, AP_WARPS * 32, 0, (cudaStream_t)stream>>>(a);
    return op_cuda(who, cudaGetLastError());
}
