// The paged key/value cache written and read back: rows of any type <-> 16-bit or 8-bit pages (mdi_kv_append, mdi_kv_read).
//
// A row is the head_dim elements of one head at one position.  8-bit rows carry one fp32 scale:
//   i8:   scale = max(absmax / 127, 2^-126), element = round-to-nearest-even(x / scale);
//   e4m3: scale = 2^k with the smallest k >= -126 such that absmax <= 448 * 2^k: x / scale is then exact in fp32, so the only
//         rounding is the one to e4m3, and a power of two loses nothing (a floating-point type keeps its relative precision).
// Rounding of i8: k = rint(x * (1 / scale)) can miss by one where x / scale is next to a half, because the reciprocal and the
// product are rounded.  The remainder x - k * scale is exact in one fma (|k| <= 127, and near a border it is a multiple of the
// operands' last place no larger than scale / 2), so comparing it with scale / 2 puts k right.
//
// Bound: bytes.  A block takes `rpb` rows of the call; a warp per row finds its sequence, slot and page; then
// groups of head_dim / 8 lanes take one row of one head each, 16 bytes a lane where the type is 16-bit, UN rows in flight.  4 x 32768 e4m3 rows of 8 x
// 128 read back as bf16 (814 MB) take 149 us, 5.5 TB/s (0.85 of the measured copy); the append of 16 ragged prompts up to 2048 bf16 rows of 8 x 128 as e4m3 15 us.
#include "ops_common.cuh"

#include <cuda_fp8.h>

#include <algorithm>

namespace mdi {
namespace {

constexpr int KR_THREADS = 256;
constexpr int KR_MAX_RPB = 64; // rows per block
constexpr int KR_UN = 2;       // rows of a head in flight per lane group (4: read back of 4 x 32768 rows 10% slower, 8: 40%)

struct KrArgs {
    OpCache c;
    OpRows k, v;
    const int *start, *pos;
    int *status;
    int n_seq, n_rows, rpb, units; // units = 2 * n_kv_head: (keys | values) x heads of one row
    unsigned units_magic;          // ceil(2^32 / units): u / units = mulhi(u, magic) for the small u of a block
};

// Where row `row` of the call, one of sequence i if of any, lives: page and row in the page.
__device__ __forceinline__ void kr_place(const KrArgs &a, int row, int i, bool read, long long &page, int &at) {
    page = -1;
    at = -1; // -1: nothing to do, -2 (read only): zeros
    if (row >= a.n_rows) return;
    const int total = a.start[a.n_seq];
    if (row >= total) return;
    const int first = a.start[i], next = a.start[i + 1];
    if (i == 0 && row < first) return;
    if (row < first || row >= next) { op_status(a.status, MDI_STATUS_RANGE); return; }
    const int slot = op_slot(a.c, i);
    const long long t = (long long)(a.pos ? a.pos[i] : 0) + (row - first);
    if (slot < 0 || t < 0 || t >= a.c.capacity) {
        op_status(a.status, MDI_STATUS_RANGE);
        if (read) at = -2;
        return;
    }
    const int p = a.c.table[(long long)slot * a.c.table_stride + (t >> a.c.page_shift)];
    if ((unsigned)p >= (unsigned)a.c.n_pages) {
        op_status(a.status, MDI_STATUS_PAGE);
        if (read) at = -2;
        return;
    }
    page = p;
    at = (int)(t & ((1 << a.c.page_shift) - 1));
}

// ---- stored types: 8 elements <-> memory ------------------------------------------------------------------------
struct StI8 { static constexpr int SIZE = 1; };
struct StE4M3 { static constexpr int SIZE = 1; };
struct StF16 { static constexpr int SIZE = 2; using T = __half; };
struct StBF16 { static constexpr int SIZE = 2; using T = __nv_bfloat16; };

// scale of a row whose largest |x| has these bits (NaN sorts above infinity, infinity above all numbers)
template <typename ST> __device__ __forceinline__ float kr_scale(unsigned big_bits);
template <> __device__ __forceinline__ float kr_scale<StI8>(unsigned b) {
    return b >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : fmaxf(__fdiv_rn(__uint_as_float(b), 127.f), 1.17549435e-38f);
}
template <> __device__ __forceinline__ float kr_scale<StE4M3>(unsigned b) {
    if (b >= 0x7f800000u) return __uint_as_float(0x7fc00000u);
    // b = 1.m * 2^(e - 127); 448 = 1.75 * 2^8: k = e - 127 - 8, one more where 1.m > 1.75 (subnormals end at k = -126 anyway)
    const int e = (int)(b >> 23), k = e - 135 + ((b & 0x7fffffu) > 0x600000u);
    return __uint_as_float((unsigned)max(k + 127, 1) << 23);
}

template <typename ST> __device__ __forceinline__ void kr_store8(unsigned char *p, const F8 &x, float scale);
template <> __device__ __forceinline__ void kr_store8<StI8>(unsigned char *p, const F8 &x, float scale) {
    const float inv = __frcp_rn(scale), half = 0.5f * scale;
    unsigned q[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float k = rintf(x.v[e] * inv);
        const float r = fmaf(-k, scale, x.v[e]);
        if (fabsf(r) >= half && (fabsf(r) > half || ((int)k & 1))) k += r > 0.f ? 1.f : -1.f;
        q[e] = (unsigned)(int)k & 0xffu;
    }
    *(uint2 *)p = make_uint2(q[0] | q[1] << 8 | q[2] << 16 | q[3] << 24, q[4] | q[5] << 8 | q[6] << 16 | q[7] << 24);
}
template <> __device__ __forceinline__ void kr_store8<StE4M3>(unsigned char *p, const F8 &x, float scale) {
    const float inv = __uint_as_float(0x7f000000u - __float_as_uint(scale)); // 2^-k: exact
    unsigned w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        w[i] = __nv_cvt_float2_to_fp8x2(make_float2(x.v[2 * i] * inv, x.v[2 * i + 1] * inv), __NV_SATFINITE, __NV_E4M3);
    *(uint2 *)p = make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
}

template <typename ST> struct StRaw { uint2 a; };
template <> struct StRaw<StF16> { uint4 a; };
template <> struct StRaw<StBF16> { uint4 a; };
template <typename ST> __device__ __forceinline__ F8 kr_unpack(const StRaw<ST> &r);
template <> __device__ __forceinline__ F8 kr_unpack<StF16>(const StRaw<StF16> &r) { return RowIO<__half>::unpack(RowIO<__half>::Raw{r.a}); }
template <> __device__ __forceinline__ F8 kr_unpack<StBF16>(const StRaw<StBF16> &r) { return RowIO<__nv_bfloat16>::unpack(RowIO<__nv_bfloat16>::Raw{r.a}); }
template <> __device__ __forceinline__ F8 kr_unpack<StI8>(const StRaw<StI8> &r) {
    F8 f;
#pragma unroll
    for (int e = 0; e < 8; ++e) f.v[e] = (float)(signed char)((e < 4 ? r.a.x : r.a.y) >> (8 * (e & 3)));
    return f;
}
template <> __device__ __forceinline__ F8 kr_unpack<StE4M3>(const StRaw<StE4M3> &r) {
    F8 f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned w = i < 2 ? r.a.x : r.a.y;
        unsigned h;
        if (i & 1) asm("{\n .reg .b16 lo, hi;\n mov.b32 {lo, hi}, %1;\n cvt.rn.f16x2.e4m3x2 %0, hi;\n}\n" : "=r"(h) : "r"(w));
        else asm("{\n .reg .b16 lo, hi;\n mov.b32 {lo, hi}, %1;\n cvt.rn.f16x2.e4m3x2 %0, lo;\n}\n" : "=r"(h) : "r"(w));
        const float2 x = __half22float2(*(const __half2 *)&h);
        f.v[2 * i] = x.x;
        f.v[2 * i + 1] = x.y;
    }
    return f;
}

template <typename RT, typename ST, int HD, bool READ>
__global__ void __launch_bounds__(KR_THREADS) k_kv_rows(const KrArgs a) {
    constexpr int LPR = HD / 8;               // lanes per row of a head
    constexpr int GROUPS = KR_THREADS / LPR;  // rows of heads a block takes at a time
    constexpr bool SCALED = ST::SIZE == 1;
    __shared__ long long s_page[KR_MAX_RPB];
    __shared__ int s_at[KR_MAX_RPB];
    const int row0 = blockIdx.x * a.rpb, tid = threadIdx.x, sub = tid % LPR, grp = tid / LPR;
    const int n_units = min(a.rpb, a.n_rows - row0) * a.units, first = blockIdx.y * GROUPS * KR_UN;
    // unit u of the block: row of the block, keys or values, head
    auto split = [&](int u, int &rl, int &which, int &h) {
        rl = (int)__umulhi((unsigned)u, a.units_magic);
        const int w = u - rl * a.units;
        which = w >= a.c.n_kv_head;
        h = w - (which ? a.c.n_kv_head : 0);
    };
    auto address = [&](int rl, int which, int h) {
        const OpRows &t = which ? a.v : a.k;
        return t.data + ((row0 + rl) * t.row_stride + h * t.head_stride + sub * 8) * (long long)sizeof(RT);
    };
    typename RowIO<RT>::Raw in[KR_UN]; // append: the rows of a round; of the first one while their places are looked up
    auto fetch = [&](int u0) {
#pragma unroll
        for (int j = 0; j < KR_UN; ++j) {
            const int u = u0 + j * GROUPS + grp;
            int rl, which, h;
            split(min(u, n_units - 1), rl, which, h);
            if (u < n_units) in[j] = RowIO<RT>::load(address(rl, which, h));
        }
    };
    if (!READ && first < n_units) fetch(first);
    for (int r = tid >> 5; r < a.rpb; r += KR_THREADS / 32) { // a warp per row: its sequence is found 32 at a time
        const int i = op_find_warp(a.start, a.n_seq, row0 + r, tid & 31);
        if ((tid & 31) == 0) kr_place(a, row0 + r, i, READ, s_page[r], s_at[r]);
    }
    __syncthreads();
    for (int u0 = first; u0 < n_units; u0 += gridDim.y * GROUPS * KR_UN) {
        long long dst[KR_UN]; // index of the row in the pool (negative: see kr_place)
        unsigned char *base[KR_UN];
#pragma unroll
        for (int j = 0; j < KR_UN; ++j) {
            const int u = u0 + j * GROUPS + grp;
            dst[j] = -1;
            if (u < n_units) {
                int rl, which, h;
                split(u, rl, which, h);
                base[j] = address(rl, which, h);
                const int at = s_at[rl];
                dst[j] = at < 0 ? at : (((s_page[rl] * 2 + which) * a.c.n_kv_head + h) << a.c.page_shift) + at;
            }
        }
        if (!READ) {
            if (u0 != first) fetch(u0);
#pragma unroll
            for (int j = 0; j < KR_UN; ++j) {
                F8 x{};
                if (dst[j] >= 0) x = RowIO<RT>::unpack(in[j]);
                unsigned char *p = a.c.pool + (dst[j] * HD + sub * 8) * ST::SIZE;
                if constexpr (SCALED) {
                    unsigned big = 0;
#pragma unroll
                    for (int e = 0; e < 8; ++e) big = max(big, __float_as_uint(x.v[e]) & 0x7fffffffu);
#pragma unroll
                    for (int o = LPR / 2; o > 0; o >>= 1) big = max(big, __shfl_xor_sync(0xffffffffu, big, o));
                    const float scale = kr_scale<ST>(big);
                    if (dst[j] >= 0) {
                        if (big >= 0x7f800000u) *(uint2 *)p = make_uint2(0, 0);
                        else kr_store8<ST>(p, x, scale);
                        if (sub == 0) a.c.scale[dst[j]] = scale;
                    }
                } else if (dst[j] >= 0) {
                    RowIO<typename ST::T>::store(p, x);
                }
            }
        } else {
            StRaw<ST> raw[KR_UN];
            float scale[KR_UN];
#pragma unroll
            for (int j = 0; j < KR_UN; ++j) {
                raw[j] = StRaw<ST>{};
                scale[j] = 1.f;
                if (dst[j] >= 0) {
                    raw[j].a = *(const decltype(raw[j].a) *)(a.c.pool + (dst[j] * HD + sub * 8) * ST::SIZE);
                    if (SCALED) scale[j] = a.c.scale[dst[j]];
                }
            }
#pragma unroll
            for (int j = 0; j < KR_UN; ++j) {
                if (dst[j] == -1) continue;
                F8 x = kr_unpack<ST>(raw[j]);
                if (SCALED) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) x.v[e] *= scale[j];
                }
                RowIO<RT>::store(base[j], x);
            }
        }
    }
}

template <typename RT, typename ST, bool READ> void kr_hd(const KrArgs &a, dim3 grid, cudaStream_t st) {
    switch (a.c.head_dim) {
        case 16: k_kv_rows<RT, ST, 16, READ><<<grid, KR_THREADS, 0, st>>>(a); break;
        case 32: k_kv_rows<RT, ST, 32, READ><<<grid, KR_THREADS, 0, st>>>(a); break;
        case 64: k_kv_rows<RT, ST, 64, READ><<<grid, KR_THREADS, 0, st>>>(a); break;
        default: k_kv_rows<RT, ST, 128, READ><<<grid, KR_THREADS, 0, st>>>(a); break;
    }
}

int kr_call(const char *who, bool read, const mdi_kv_cache *cache, int n_seq, const int32_t *slot_dev, const int32_t *seq_start_dev,
            const int32_t *pos_dev, int n_rows, const mdi_rows *k, const mdi_rows *v, int32_t *status_dev, void *stream) {
    int rc = op_check_cache(who, cache);
    if (rc != MDI_OK) return rc;
    if (n_seq < 0 || n_rows < 0) return op_fail(MDI_ERR_ARG, "%s: negative n_seq or n_rows", who);
    if (!slot_dev && n_seq > cache->n_slots) return op_fail(MDI_ERR_ARG, "%s: %d sequences, but the page table has %d slots", who, n_seq, cache->n_slots);
    if ((rc = op_check_rows(who, "k", k, n_rows, cache->n_kv_head, read)) != MDI_OK) return rc;
    if ((rc = op_check_rows(who, "v", v, n_rows, cache->n_kv_head, read)) != MDI_OK) return rc;
    if (k->dtype != v->dtype) return op_fail(MDI_ERR_ARG, "%s: k and v differ in dtype", who);
    if ((rc = op_check_ptrs(who, {{"pool_dev", cache->pool_dev, false}, {"scale_dev", cache->scale_dev, !op_scaled(cache)}, {"page_table_dev", cache->page_table_dev, false},
                                  {"k", k->data_dev, n_rows == 0}, {"v", v->data_dev, n_rows == 0}, {"slot_dev", slot_dev, true},
                                  {"seq_start_dev", seq_start_dev, false}, {"pos_dev", pos_dev, read || n_seq == 0}, {"status_dev", status_dev, true}})) != MDI_OK)
        return rc;
    if (n_seq == 0 || n_rows == 0) return MDI_OK;
    KrArgs a{};
    a.c = op_cache(cache, slot_dev);
    a.k = op_rows(k); a.v = op_rows(v);
    a.start = seq_start_dev; a.pos = pos_dev; a.status = status_dev;
    a.n_seq = n_seq; a.n_rows = n_rows;
    a.units = 2 * cache->n_kv_head;
    a.units_magic = (unsigned)(((1ull << 32) + a.units - 1) / a.units);
    // A block's share: rounds of its lane groups, UN rows each.  Finding a row's place takes a chain of dependent loads, so where
    // there is work for every SM several times over a block takes more rows (4 x 32768 rows of 8 x 128: 1, 2, 4 rounds 168, 155,
    // 150 us); where there is not, fewer, and there are more blocks (64 rows of 32 x 128: 7.4, 7.6, 11 us).
    const int groups = KR_THREADS / (cache->head_dim / 8) * KR_UN;
    const int64_t passes = (int64_t)n_rows * a.units / groups;
    const int rounds = passes >= 4 * 148 * 8 ? 4 : passes >= 148 * 8 ? 2 : 1;
    a.rpb = std::max(1, std::min(KR_MAX_RPB, groups * rounds / a.units));
    const dim3 grid((n_rows + a.rpb - 1) / a.rpb, std::max(1, std::min(64, (a.rpb * a.units + groups * rounds - 1) / (groups * rounds))));
    cudaStream_t st = (cudaStream_t)stream;
#define KR_GO(ST)                                                                  \
    do {                                                                           \
        if (read) OP_ROW_DISPATCH(k->dtype, (kr_hd<RT, ST, true>(a, grid, st)));   \
        else OP_ROW_DISPATCH(k->dtype, (kr_hd<RT, ST, false>(a, grid, st)));       \
    } while (0)
    switch (cache->dtype) {
        case MDI_KV_I8: KR_GO(StI8); break;
        case MDI_KV_E4M3: KR_GO(StE4M3); break;
        case MDI_KV_F16: KR_GO(StF16); break;
        default: KR_GO(StBF16); break;
    }
#undef KR_GO
    return op_cuda(who, cudaGetLastError());
}

} // namespace
} // namespace mdi

extern "C" int mdi_kv_append(const mdi_kv_cache *cache, int n_seq, const int32_t *slot_dev, const int32_t *seq_start_dev, const int32_t *pos_dev,
                             int n_rows, const mdi_rows *k, const mdi_rows *v, int32_t *status_dev, void *stream) {
    return mdi::kr_call("mdi_kv_append", false, cache, n_seq, slot_dev, seq_start_dev, pos_dev, n_rows, k, v, status_dev, stream);
}

extern "C" int mdi_kv_read(const mdi_kv_cache *cache, int n_seq, const int32_t *slot_dev, const int32_t *seq_start_dev, const int32_t *pos_dev,
                           int n_rows, const mdi_rows *k_out, const mdi_rows *v_out, int32_t *status_dev, void *stream) {
    return mdi::kr_call("mdi_kv_read", true, cache, n_seq, slot_dev, seq_start_dev, pos_dev, n_rows, k_out, v_out, status_dev, stream);
}
