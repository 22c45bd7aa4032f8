// Shared by the operators on the caller's own device memory (kv_rows.cu, attn_decode.cu, attn_prompt.cu): the checks of
// their arguments, what a kernel needs to know of a paged cache, and row types.
#pragma once
#include "mdi.h"

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <atomic>
#include <initializer_list>
#include <stdint.h>

void mdi_internal_set_error(const char *text); // mdi.cu: text returned by mdi_last_error(NULL)

namespace mdi {

// ---- host: checks.  Each returns MDI_OK or an error code whose text has been set. -------------------------------
int op_fail(int code, const char *fmt, ...);
int op_cuda(const char *who, cudaError_t e); // MDI_OK for cudaSuccess
struct OpPtr { const char *name; const void *p; bool optional; };
// every pointer must be device memory of the current device (null passes only where `optional`); checked last
int op_check_ptrs(const char *who, std::initializer_list<OpPtr> ptrs);
// a row view of `rows` rows of `heads` heads: type, alignment, strides (those of a dimension of size 1 do not matter; a zero one repeats an input, and is refused where `written`)
int op_check_rows(const char *who, const char *name, const mdi_rows *r, int rows, int heads, bool written);
int op_check_cache(const char *who, const mdi_kv_cache *c);
inline bool op_scaled(const mdi_kv_cache *c) { return c->dtype == MDI_KV_I8 || c->dtype == MDI_KV_E4M3; }

// Runs a call once per device and place of use (setting a kernel's shared memory costs as much as its launch).
struct OpOnce {
    std::atomic<uint64_t> done{0}; // a bit per device
    template <typename F> cudaError_t operator()(F f) {
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return e;
        if (dev < 64 && (done.load(std::memory_order_acquire) >> dev & 1)) return cudaSuccess;
        if ((e = f()) == cudaSuccess && dev < 64) done.fetch_or(1ull << dev, std::memory_order_release);
        return e;
    }
};

// ---- device view of a paged cache ------------------------------------------------------------------------------
struct OpCache {
    unsigned char *pool;
    float *scale;
    const int *table;
    const int *slot; // page-table row of each sequence, or null: the sequence's number
    long long table_stride;
    int n_pages, n_slots, pages_per_seq, page_shift, n_kv_head, head_dim;
    long long capacity; // rows a slot can hold
};
OpCache op_cache(const mdi_kv_cache *c, const int32_t *slot_dev);

struct OpRows {
    unsigned char *data;
    long long row_stride, head_stride; // elements
};
inline OpRows op_rows(const mdi_rows *r) { return OpRows{(unsigned char *)r->data_dev, r->row_stride, r->head_stride}; }

__device__ __forceinline__ void op_status(int *status, int bit) {
    if (status) atomicOr(status, bit);
}
// page-table row of sequence i (negative: none)
__device__ __forceinline__ int op_slot(const OpCache &c, int i) {
    const int s = c.slot ? c.slot[i] : i;
    return (unsigned)s < (unsigned)c.n_slots ? s : -1;
}
// Last sequence i of [0, n_seq) with start[i] <= row (start ascends; the caller checks start[i] <= row < start[i + 1]).  All lanes of
// a warp: each round looks at 32 places at once, so that up to 1024 sequences take two dependent loads.
__device__ __forceinline__ int op_find_warp(const int *start, int n_seq, int row, int lane) {
    int lo = 0, n = n_seq;
    while (n > 1) {
        const int step = (n + 31) / 32, i = lane * step;
        const unsigned at = __ballot_sync(0xffffffffu, i < n && start[lo + min(i, n - 1)] <= row);
        const int k = at ? 31 - __clz(at) : 0;
        lo += k * step;
        n = min(step, n - k * step);
    }
    return lo;
}
// ---- 8 elements of a row ---------------------------------------------------------------------------------------
struct F8 { float v[8]; };

template <typename T> struct RowIO;
template <> struct RowIO<float> {
    struct Raw { float4 a, b; };
    static __device__ __forceinline__ Raw load(const unsigned char *p) { return Raw{__ldg((const float4 *)p), __ldg((const float4 *)p + 1)}; }
    static __device__ __forceinline__ F8 unpack(const Raw &r) { return F8{{r.a.x, r.a.y, r.a.z, r.a.w, r.b.x, r.b.y, r.b.z, r.b.w}}; }
    static __device__ __forceinline__ void store(unsigned char *p, const F8 &f) {
        ((float4 *)p)[0] = make_float4(f.v[0], f.v[1], f.v[2], f.v[3]);
        ((float4 *)p)[1] = make_float4(f.v[4], f.v[5], f.v[6], f.v[7]);
    }
};
template <> struct RowIO<__half> {
    struct Raw { uint4 a; };
    static __device__ __forceinline__ Raw load(const unsigned char *p) { return Raw{__ldg((const uint4 *)p)}; }
    static __device__ __forceinline__ F8 unpack(const Raw &r) {
        F8 f;
        const __half2 *h = (const __half2 *)&r.a;
#pragma unroll
        for (int i = 0; i < 4; ++i) { const float2 x = __half22float2(h[i]); f.v[2 * i] = x.x; f.v[2 * i + 1] = x.y; }
        return f;
    }
    static __device__ __forceinline__ void store(unsigned char *p, const F8 &f) {
        uint4 r;
        __half2 *h = (__half2 *)&r;
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = __floats2half2_rn(f.v[2 * i], f.v[2 * i + 1]);
        *(uint4 *)p = r;
    }
};
template <> struct RowIO<__nv_bfloat16> {
    struct Raw { uint4 a; };
    static __device__ __forceinline__ Raw load(const unsigned char *p) { return Raw{__ldg((const uint4 *)p)}; }
    static __device__ __forceinline__ F8 unpack(const Raw &r) {
        F8 f;
        const uint32_t w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { f.v[2 * i] = __uint_as_float(w[i] << 16); f.v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
        return f;
    }
    static __device__ __forceinline__ void store(unsigned char *p, const F8 &f) {
        uint4 r;
        __nv_bfloat162 *h = (__nv_bfloat162 *)&r;
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(f.v[2 * i], f.v[2 * i + 1]);
        *(uint4 *)p = r;
    }
};

// Calls `call` with RT bound to the element type of MDI_DTYPE_* code `dt`.
#define OP_ROW_DISPATCH(dt, call)                                          \
    do {                                                                   \
        if ((dt) == MDI_DTYPE_F32) { using RT = float; call; }             \
        else if ((dt) == MDI_DTYPE_F16) { using RT = __half; call; }       \
        else { using RT = __nv_bfloat16; call; }                           \
    } while (0)

} // namespace mdi
