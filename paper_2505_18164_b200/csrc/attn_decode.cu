// Attention of one new token per sequence over a paged key/value cache (mdi_attn_decode):
//     out[i][h] = sum_j softmax_j(scale * q[i][h] . K_j) V_j,   j < len[i],   K, V of key/value head h / group.
//
// Bound: the bytes of the cached rows.  What the layout is for:
//  * Work is cut into tiles of 16 cached rows (a tile never crosses a page).  All tiles of all (sequence, key/value head,
//    chunk of up to 8 of its query heads) are laid end to end and dealt to the warps of the launch in equal contiguous
//    shares, so sequences of any mix of lengths keep every warp equally busy.  A (sequence, head) that a share boundary
//    cuts leaves partial results (maximum, sum, unnormalised output) in the workspace; a second, small kernel joins them in
//    a fixed order.  Nothing depends on timing.
//  * A warp streams its tiles through its own ring of shared memory with asynchronous copies: every lane copies exactly the
//    bytes that it will use itself as matrix-instruction fragments, so a stage needs no barrier.
//  * Products run on the tensor cores (mma.sync m16n8k16, fp32 accumulators), not for their rate but because one
//    instruction then serves the up to 8 query heads that share the row.  Scores: A = query (rows 0-7 the heads' high
//    parts, rows 8-15 their low parts), B = 8 cached rows; a lane then holds the scores of head lane / 4 for cached rows
//    2 (lane % 4), + 1, which is the layout that the B operand of the second product wants: A = V transposed (16 elements of
//    head_dim x 16 rows), B = weights.  Elements of head_dim and rows are assigned to fragment positions so that all copies
//    are wide and contiguous; both operands of a product use the same assignment.
//  * 8-bit elements become fp16 exactly in registers (int8: a byte under the exponent of 1024, minus 1152).  Scales stay
//    outside of the products: the key's multiplies the score, the value's the weight.
//  * Rounding: queries and weights are used as two 16-bit planes (high + low, 16 to 22 bits together; queries scaled by a
//    power of two per head, weights by a power of two that follows the largest value scale seen, so that fp16's range does
//    not matter); scores, maximum, sums and outputs are fp32.
#include "ops_common.cuh"

#include <cuda_fp8.h>

#include <algorithm>
#include <type_traits>

namespace mdi {
namespace {

constexpr int AD_WARPS = 4;      // warps per block (they share nothing but the table of lengths)
constexpr int AD_THREADS = AD_WARPS * 32;
constexpr int AD_STAGES = 3;
constexpr int AD_MAX_SEQ = 256;  // sequences per launch (their table shares shared memory with the rings of 4 blocks per SM)
constexpr int AD_HC = 8;         // query heads per chunk
constexpr int AD_SM = 148;
constexpr float AD_SLACK = 4.f;  // a maximum may be exceeded by 2^4 before what has been summed is rescaled
constexpr int AD_MERGE_THREADS = 128;

struct AdArgs {
    OpCache c;
    OpRows q, out;
    const int *len;
    int *status;
    long long *head;  // workspace: tiles before each sequence, [n_seq + 1]
    float *part;      // workspace: [warps][2][hc][HD + 4]: output, then maximum, sum, exponent of the weights' scale
    int n_seq, seq0;  // sequences of this launch, first one's number
    int n_head, group, chunks, hc, n_warps, min_tiles;
    float scale_log2e;
};

enum { AD_I8, AD_E4M3, AD_F16, AD_BF16 };
template <int ST> struct AdStore {
    static constexpr int SIZE = ST <= AD_E4M3 ? 1 : 2;
    static constexpr bool SCALED = SIZE == 1, BF = ST == AD_BF16;
    static constexpr int BLOCKS = SIZE == 1 ? 4 : 2; // resident blocks per SM
};

__device__ __forceinline__ void ad_mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, std::false_type) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ad_mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, std::true_type) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float ad_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float ad_pow2(int e) { return __uint_as_float((unsigned)(e + 127) << 23); } // -126 <= e <= 127

__device__ __forceinline__ void ad_load4(float (&f)[4], const float *p) {
    const float4 v = *(const float4 *)p;
    f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
}
__device__ __forceinline__ void ad_load4(float (&f)[4], const __half *p) {
    const uint2 v = *(const uint2 *)p;
    const float2 a = __half22float2(*(const __half2 *)&v.x), b = __half22float2(*(const __half2 *)&v.y);
    f[0] = a.x; f[1] = a.y; f[2] = b.x; f[3] = b.y;
}
__device__ __forceinline__ void ad_load4(float (&f)[4], const __nv_bfloat16 *p) {
    const uint2 v = *(const uint2 *)p;
    f[0] = __uint_as_float(v.x << 16); f[1] = __uint_as_float(v.x & 0xffff0000u);
    f[2] = __uint_as_float(v.y << 16); f[3] = __uint_as_float(v.y & 0xffff0000u);
}

// x, y as high and low 16-bit planes
__device__ __forceinline__ void ad_split(float x, float y, uint32_t &hi, uint32_t &lo, std::false_type) {
    const __half2 h = __floats2half2_rn(x, y);
    const float2 f = __half22float2(h);
    const __half2 l = __floats2half2_rn(x - f.x, y - f.y);
    hi = *(const uint32_t *)&h;
    lo = *(const uint32_t *)&l;
}
__device__ __forceinline__ void ad_split(float x, float y, uint32_t &hi, uint32_t &lo, std::true_type) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
    hi = *(const uint32_t *)&h;
    const __nv_bfloat162 l = __floats2bfloat162_rn(x - __uint_as_float(hi << 16), y - __uint_as_float(hi & 0xffff0000u));
    lo = *(const uint32_t *)&l;
}

// Two stored 8-bit elements (the bytes `sel` picks from w: 0x4140 the lower two, 0x4342 the upper two) as fp16.
template <int ST, int UPPER> __device__ __forceinline__ uint32_t ad_wide(uint32_t w) {
    if constexpr (ST == AD_I8) { // w: biased by 128
        const uint32_t h = __byte_perm(w, 0x64646464u, UPPER ? 0x4342 : 0x4140); // 1024 + (x + 128)
        const __half2 r = __hsub2(*(const __half2 *)&h, __half2half2(__ushort_as_half(0x6480))); // - 1152
        return *(const uint32_t *)&r;
    } else {
        const __half2_raw r = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(UPPER ? w >> 16 : w & 0xffffu), __NV_E4M3);
        return (uint32_t)r.x | (uint32_t)r.y << 16;
    }
}
template <int ST> __device__ __forceinline__ uint32_t ad_bias(uint32_t w) { return ST == AD_I8 ? w ^ 0x80808080u : w; }

// `bytes` (2, 4, 8 or 16) from global to shared memory, zeros where !ok
template <int BYTES> __device__ __forceinline__ void ad_copy(uint32_t dst, const unsigned char *src, bool ok) {
    const int n = ok ? BYTES : 0;
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
    else if constexpr (BYTES == 8) asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
    else if constexpr (BYTES == 4) asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
    else {
        const unsigned short v = ok ? *(const unsigned short *)src : (unsigned short)0;
        asm volatile("st.shared.u16 [%0], %1;" ::"r"(dst), "h"(v) : "memory");
    }
}
template <int BYTES> __device__ __forceinline__ void ad_read(uint32_t (&w)[(BYTES + 3) / 4], uint32_t src) {
    if constexpr (BYTES == 16) asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(src) : "memory");
    else if constexpr (BYTES == 8) asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(src) : "memory");
    else if constexpr (BYTES == 4) asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[0]) : "r"(src) : "memory");
    else {
        unsigned short v;
        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(src) : "memory");
        w[0] = v;
    }
}

// How a tile's 16 rows of keys and values are dealt to lanes, g = lane / 4, t = lane % 4.  Keys: lane holds of rows g and
// g + 8 the chunks t, t + 4, ... of KC bytes.  Values: of rows 2t, 2t + 1, 2t + 8, 2t + 9 the chunks g, g + 8, ... of VC bytes.
template <int ST, int HD> struct AdTile {
    static constexpr int SZ = AdStore<ST>::SIZE;
    static constexpr int KB = HD * SZ / 4, KC = KB < 16 ? KB : 16, KN = KB / KC; // bytes per lane and row, chunk, chunks
    static constexpr int VB = HD * SZ / 8, VC = VB < 16 ? VB : 16, VN = VB / VC;
    static constexpr int VSLOT = VC < 4 ? 4 : VC;                                // 2-byte chunks sit in words of their own
    static constexpr int K_BYTES = 2 * KN * KC * 32, V_BYTES = 4 * VN * VSLOT * 32;
    static constexpr int SCALES = K_BYTES + V_BYTES, LIVE = SCALES + (SZ == 1 ? 128 : 0); // then the 32 scales and the number of rows
    static constexpr int STAGE = LIVE + 16;
    static constexpr int KE = KC / SZ, VE = VC / SZ;                             // elements per chunk
    static __device__ __forceinline__ int k_dim(int t, int s) { const int e = 4 * s; return e / KE * (4 * KE) + t * KE + e % KE; } // first of a lane's 4 elements of k-step s
    static __device__ __forceinline__ int v_dim(int g, int j) { return j / VE * (8 * VE) + g * VE + j % VE; }                      // a lane's j-th element
};
template <int ST, int HD> constexpr size_t ad_smem() { return (size_t)AD_WARPS * AD_STAGES * AdTile<ST, HD>::STAGE + (AD_MAX_SEQ + 1) * 8 + AD_MAX_SEQ * 4; }

__device__ __forceinline__ int ad_len(const AdArgs &a, int i, int *status) {
    const int n = a.len[i], slot = a.c.slot ? a.c.slot[i] : a.seq0 + i;
    if ((unsigned)slot >= (unsigned)a.c.n_slots || n < 0) { op_status(status, MDI_STATUS_RANGE); return 0; }
    if (n > a.c.capacity) { op_status(status, MDI_STATUS_RANGE); return (int)a.c.capacity; }
    return n;
}

// Where in the line of tiles: sequence, (head, chunk) pair within it, tile within the pair
struct AdCursor {
    int i, pair, tile, n_tiles, len;
    __device__ __forceinline__ void enter(const int *s_len, int seq) { i = seq; len = s_len[seq]; n_tiles = (len + 15) >> 4; }
    __device__ __forceinline__ void seek(const long long *pref, const int *s_len, int n_seq, int pairs, long long at) {
        int lo = 0, hi = n_seq - 1; // last sequence whose first tile is at or before `at`
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (pref[mid] * pairs <= at) lo = mid; else hi = mid - 1;
        }
        enter(s_len, lo);
        const long long in = at - pref[lo] * pairs;
        pair = (int)(in / n_tiles);
        tile = (int)(in - (long long)pair * n_tiles);
    }
    // true: the next tile belongs to another pair
    __device__ __forceinline__ bool advance(const int *s_len, int n_seq, int pairs) {
        if (++tile < n_tiles) return false;
        tile = 0;
        if (++pair == pairs) {
            pair = 0;
            do ++i; while (i < n_seq && s_len[i] == 0);
            if (i < n_seq) enter(s_len, i);
        }
        return true;
    }
};

// share of warp w: tiles [T w / W, T (w + 1) / W)
__device__ __forceinline__ long long ad_share(long long T, int W, int w) { return T * w / W; }
__device__ __forceinline__ int ad_warps(const AdArgs &a, long long T) {
    const long long w = T / a.min_tiles;
    return (int)(w < 1 ? 1 : w < a.n_warps ? w : a.n_warps);
}

template <typename RT, int ST, int HD>
__global__ void __launch_bounds__(AD_THREADS, AdStore<ST>::BLOCKS) k_attn_decode_op(const AdArgs a) {
    using TL = AdTile<ST, HD>;
    using BF = std::integral_constant<bool, AdStore<ST>::BF>;
    constexpr bool SCALED = AdStore<ST>::SCALED;
    constexpr int KS = HD / 16;                       // k-steps of the scores, m-tiles of the output
    constexpr float PUP = AdStore<ST>::BF ? 1.f : 1024.f; // fp16 weights: at most 2^4 * 2 * 2^10
    extern __shared__ __align__(16) unsigned char ad_raw[];
    long long *s_pref = (long long *)(ad_raw + AD_WARPS * AD_STAGES * TL::STAGE);
    int *s_len = (int *)(s_pref + AD_MAX_SEQ + 1);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    // ---- lengths, tiles before each sequence (every block for itself; block 0 leaves them for the joining kernel)
    {
        __shared__ long long s_sum[AD_WARPS];
        long long run = 0;
        for (int base = 0; base < a.n_seq; base += AD_THREADS) {
            const int i = base + tid;
            const int n = i < a.n_seq ? ad_len(a, i, blockIdx.x == 0 ? a.status : nullptr) : 0;
            const long long mine = (n + 15) >> 4;
            long long incl = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long up = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += up;
            }
            if (lane == 31) s_sum[warp] = incl;
            __syncthreads();
            long long before = run;
            for (int w = 0; w < AD_WARPS; ++w) { if (w < warp) before += s_sum[w]; run += s_sum[w]; }
            if (i < a.n_seq) {
                s_len[i] = n;
                s_pref[i] = before + incl - mine;
                if (blockIdx.x == 0) a.head[i] = before + incl - mine;
            }
            __syncthreads();
        }
        if (tid == 0) {
            s_pref[a.n_seq] = run;
            if (blockIdx.x == 0) a.head[a.n_seq] = run;
        }
        __syncthreads();
    }
    const int pairs = a.c.n_kv_head * a.chunks;
    const long long T = s_pref[a.n_seq] * pairs;
    const int W = ad_warps(a, T), w = blockIdx.x * AD_WARPS + warp;
    if (T == 0 || w >= W) return;
    const long long first = ad_share(T, W, w), last = ad_share(T, W, w + 1);
    long long left = last - first; // tiles still to compute

    AdCursor cur, nxt; // consumer, producer
    cur.seek(s_pref, s_len, a.n_seq, pairs, first);
    nxt = cur;
    long long to_load = left;
    int batch_i = -1, batch_tile = 0, batch_page = -1, page_slot = 0;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(ad_raw) + warp * AD_STAGES * TL::STAGE;
    const long long head_rows = (long long)a.c.n_kv_head << a.c.page_shift; // rows of one half of a page

    // The next tile into stage `s`.  The lanes hold the page numbers of the next 32 tiles; the rows of a page that does not exist
    // count as behind the end.
    auto load = [&](int s) {
        if (to_load > 0) {
            --to_load;
            if (batch_i != nxt.i || nxt.tile < batch_tile || nxt.tile >= batch_tile + 32) {
                batch_i = nxt.i;
                batch_tile = nxt.tile;
                page_slot = a.c.slot ? a.c.slot[nxt.i] : a.seq0 + nxt.i;
                batch_page = -1;
                if (batch_tile + lane < nxt.n_tiles) {
                    batch_page = __ldg(a.c.table + (long long)page_slot * a.c.table_stride + ((long long)(batch_tile + lane) << 4 >> a.c.page_shift));
                    if ((unsigned)batch_page >= (unsigned)a.c.n_pages) { op_status(a.status, MDI_STATUS_PAGE); batch_page = -1; }
                }
            }
            const int page = __shfl_sync(0xffffffffu, batch_page, nxt.tile - batch_tile);
            const int row0 = nxt.tile << 4, rows = page < 0 ? 0 : min(16, nxt.len - row0);
            const int h = a.chunks == 1 ? nxt.pair : nxt.pair / a.chunks;
            const long long kr = (page < 0 ? 0 : ((((long long)page * 2) * a.c.n_kv_head + h) << a.c.page_shift) + (row0 & ((1 << a.c.page_shift) - 1)));
            const unsigned char *kp = a.c.pool + kr * (HD * TL::SZ), *vp = kp + head_rows * (HD * TL::SZ);
            const uint32_t st = ring + s * TL::STAGE;
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int c = 0; c < TL::KN; ++c)
                    ad_copy<TL::KC>(st + ((r * TL::KN + c) * 32 + lane) * TL::KC, kp + (8 * r + g) * (HD * TL::SZ) + (c * 4 + t) * TL::KC, 8 * r + g < rows);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 2 * t + (r & 1) + (r >> 1) * 8;
#pragma unroll
                for (int c = 0; c < TL::VN; ++c)
                    ad_copy<TL::VC>(st + TL::K_BYTES + ((r * TL::VN + c) * 32 + lane) * TL::VSLOT, vp + row * (HD * TL::SZ) + (c * 8 + g) * TL::VC, row < rows);
            }
            if (SCALED) { // lanes 0-15 the keys' scales, 16-31 the values'
                const int row = lane & 15;
                ad_copy<4>(st + TL::SCALES + lane * 4, (const unsigned char *)(a.c.scale + kr + (lane >> 4) * head_rows + row), row < rows);
            }
            if (lane == 0) asm volatile("st.shared.s32 [%0], %1;" ::"r"(st + TL::LIVE), "r"(rows) : "memory");
            nxt.advance(s_len, a.n_seq, pairs);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };

#pragma unroll
    for (int s = 0; s < AD_STAGES - 1; ++s) load(s);

    uint32_t qa[KS][4];
    float o[KS][4], m = -INFINITY, l = 0.f, q_up = 1.f, v_inv = 1.f;
    int v_exp = 0;
    bool fresh = true, first_seg = true;
    int stage = 0;
    while (left > 0) {
        if (fresh) { // a new (sequence, head, chunk): its queries, scaled into log2 units, as fragments
            fresh = false;
            const int h = cur.pair / a.chunks, ch = cur.pair - h * a.chunks;
            const int qh = h * a.group + ch * AD_HC + g;
            const bool there = ch * AD_HC + g < a.group;
            const RT *q = (const RT *)a.q.data + cur.i * a.q.row_stride + (there ? qh : 0) * a.q.head_stride;
            float f[KS][4];
            unsigned big = 0;
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int e = 0; e < 4; ++e) f[s][e] = 0.f;
#pragma unroll
            for (int s = 0; s < KS; ++s)
                if (there) ad_load4(f[s], q + TL::k_dim(t, s));
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    f[s][e] *= a.scale_log2e;
                    big = max(big, __float_as_uint(f[s][e]) & 0x7fffffffu);
                }
            q_up = 1.f;
            float q_down = 1.f;
            if (!AdStore<ST>::BF) { // fp16 planes: the largest element to [1, 2)
                big = max(big, __shfl_xor_sync(0xffffffffu, big, 1));
                big = max(big, __shfl_xor_sync(0xffffffffu, big, 2));
                if (big != 0 && big < 0x7f800000u) {
                    const int e = min(max((int)(big >> 23) - 127, -126), 126);
                    q_up = ad_pow2(e);
                    q_down = ad_pow2(-e);
                }
            }
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                ad_split(f[s][0] * q_down, f[s][1] * q_down, qa[s][0], qa[s][1], BF());
                ad_split(f[s][2] * q_down, f[s][3] * q_down, qa[s][2], qa[s][3], BF());
#pragma unroll
                for (int e = 0; e < 4; ++e) o[s][e] = 0.f;
            }
            m = -INFINITY;
            l = 0.f;
            v_exp = SCALED ? -126 : 0;
            v_inv = SCALED ? ad_pow2(126) : 1.f;
        }
        asm volatile("cp.async.wait_group %0;" ::"n"(AD_STAGES - 2) : "memory");
        __syncwarp();
        load(stage == 0 ? AD_STAGES - 1 : stage - 1); // the stage that the previous tile used
        const uint32_t st = ring + stage * TL::STAGE;
        stage = stage == AD_STAGES - 1 ? 0 : stage + 1;

        // ---- scores of 16 rows
        float s[2][4];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
#pragma unroll
            for (int e = 0; e < 4; ++e) s[r][e] = 0.f;
            uint32_t kw[TL::KN][(TL::KC + 3) / 4];
#pragma unroll
            for (int c = 0; c < TL::KN; ++c) ad_read<TL::KC>(kw[c], st + ((r * TL::KN + c) * 32 + lane) * TL::KC);
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                uint32_t b0, b1;
                if constexpr (TL::SZ == 1) {
                    const uint32_t x = ad_bias<ST>(kw[k * 4 / TL::KC][k * 4 % TL::KC / 4]);
                    b0 = ad_wide<ST, 0>(x);
                    b1 = ad_wide<ST, 1>(x);
                } else {
                    b0 = kw[k * 8 / TL::KC][k * 8 % TL::KC / 4];
                    b1 = kw[k * 8 / TL::KC][k * 8 % TL::KC / 4 + 1];
                }
                ad_mma(s[r], qa[k], b0, b1, BF());
            }
        }
        float2 vs[2] = {make_float2(1.f, 1.f), make_float2(1.f, 1.f)};
        float x[4];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            float2 ks = make_float2(q_up, q_up);
            if (SCALED) {
                const uint32_t sc = st + TL::SCALES + (8 * r + 2 * t) * 4;
                asm volatile("ld.shared.v2.f32 {%0,%1}, [%2];" : "=f"(ks.x), "=f"(ks.y) : "r"(sc) : "memory");
                asm volatile("ld.shared.v2.f32 {%0,%1}, [%2];" : "=f"(vs[r].x), "=f"(vs[r].y) : "r"(sc + 64) : "memory");
                ks.x *= q_up;
                ks.y *= q_up;
            }
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                float sum = s[r][b] + s[r][2 + b];
                // a 16-bit key may be infinite: the low part of the query, of either sign or zero, has no say then
                if (!SCALED && fabsf(s[r][b]) == INFINITY) sum = s[r][b];
                x[2 * r + b] = sum * (b ? ks.y : ks.x);
            }
        }
        // ---- rows behind the end, or of a page that does not exist
        {
            int live;
            asm volatile("ld.shared.s32 %0, [%1];" : "=r"(live) : "r"(st + TL::LIVE) : "memory");
            if (live < 16) {
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    if (8 * r + 2 * t >= live) { x[2 * r] = -INFINITY; vs[r].x = 0.f; }
                    if (8 * r + 2 * t + 1 >= live) { x[2 * r + 1] = -INFINITY; vs[r].y = 0.f; }
                }
            }
        }
        // ---- running maximum; the sums so far follow it only when it rises by more than the slack
        float top = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        int e_new = v_exp;
        if (SCALED) {
            float big = fmaxf(fmaxf(vs[0].x, vs[0].y), fmaxf(vs[1].x, vs[1].y));
            big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
            big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
            e_new = max(v_exp, min((int)(__float_as_uint(big) >> 23) - 127, 126)); // scales are positive
        }
        const bool rise = top > m + AD_SLACK || (m == -INFINITY && top > -INFINITY);
        if (__any_sync(0xffffffffu, rise || e_new != v_exp)) {
            const float mn = rise ? top : m;
            float f = rise ? (m == -INFINITY ? 0.f : ad_exp2(m - mn)) : 1.f;
            l *= f;
            m = mn;
            if (SCALED) {
                f *= v_exp - e_new >= -126 ? ad_pow2(v_exp - e_new) : 0.f;
                v_exp = e_new;
                v_inv = ad_pow2(-e_new);
            }
            const float f0 = __shfl_sync(0xffffffffu, f, 8 * t), f1 = __shfl_sync(0xffffffffu, f, 8 * t + 4); // heads 2t, 2t + 1
#pragma unroll
            for (int k = 0; k < KS; ++k) { o[k][0] *= f0; o[k][1] *= f1; o[k][2] *= f0; o[k][3] *= f1; }
        }
        const float ref = m == -INFINITY ? 0.f : m;
        uint32_t ph[2], pl[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const float p0 = ad_exp2(x[2 * r] - ref), p1 = ad_exp2(x[2 * r + 1] - ref);
            l += p0 + p1;
            if (SCALED) ad_split(p0 * PUP * (vs[r].x * v_inv), p1 * PUP * (vs[r].y * v_inv), ph[r], pl[r], BF());
            else ad_split(p0 * PUP, p1 * PUP, ph[r], pl[r], BF());
        }
        // ---- values
        uint32_t vw[4][TL::VN][(TL::VC + 3) / 4];
#pragma unroll
        for (int c = 0; c < TL::VN; ++c) {
#pragma unroll
            for (int r = 0; r < 4; ++r) ad_read<TL::VC>(vw[r][c], st + TL::K_BYTES + ((r * TL::VN + c) * 32 + lane) * TL::VSLOT);
#pragma unroll
            for (int i = 0; i < (TL::VC + 3) / 4; ++i) {
                uint32_t av[4];
                if constexpr (TL::SZ == 1) {
                    const uint32_t x0 = ad_bias<ST>(vw[0][c][i]), x1 = ad_bias<ST>(vw[1][c][i]), x2 = ad_bias<ST>(vw[2][c][i]), x3 = ad_bias<ST>(vw[3][c][i]);
                    constexpr int WORDS = (TL::VC + 3) / 4;
                    const int k = (c * WORDS + i) * 2; // a word holds the elements of two m-tiles
                    uint32_t y = __byte_perm(x0, x1, 0x5140), z = __byte_perm(x2, x3, 0x5140);
                    av[0] = ad_wide<ST, 0>(y); av[1] = ad_wide<ST, 1>(y); av[2] = ad_wide<ST, 0>(z); av[3] = ad_wide<ST, 1>(z);
                    ad_mma(o[k], av, ph[0], ph[1], BF());
                    ad_mma(o[k], av, pl[0], pl[1], BF());
                    if constexpr (TL::VC >= 4) {
                        y = __byte_perm(x0, x1, 0x7362); z = __byte_perm(x2, x3, 0x7362);
                        av[0] = ad_wide<ST, 0>(y); av[1] = ad_wide<ST, 1>(y); av[2] = ad_wide<ST, 0>(z); av[3] = ad_wide<ST, 1>(z);
                        ad_mma(o[k + 1], av, ph[0], ph[1], BF());
                        ad_mma(o[k + 1], av, pl[0], pl[1], BF());
                    }
                } else {
                    const int k = c * (TL::VC / 4) + i;
                    av[0] = __byte_perm(vw[0][c][i], vw[1][c][i], 0x5410);
                    av[1] = __byte_perm(vw[0][c][i], vw[1][c][i], 0x7632);
                    av[2] = __byte_perm(vw[2][c][i], vw[3][c][i], 0x5410);
                    av[3] = __byte_perm(vw[2][c][i], vw[3][c][i], 0x7632);
                    ad_mma(o[k], av, ph[0], ph[1], BF());
                    ad_mma(o[k], av, pl[0], pl[1], BF());
                }
            }
        }
        // ---- the end of this pair, or of this warp's share of it
        --left;
        const AdCursor was = cur;
        const bool turn = cur.advance(s_len, a.n_seq, pairs);
        if (!turn && left > 0) continue;
        fresh = true;
        l += __shfl_xor_sync(0xffffffffu, l, 1);
        l += __shfl_xor_sync(0xffffffffu, l, 2);
        // this warp holds all of the pair if it began at its first tile (its share begins there or it came from another pair)
        const long long pair_first = s_pref[was.i] * pairs + (long long)was.pair * was.n_tiles;
        const bool whole = turn && (!first_seg || pair_first >= first);
        const int h = was.pair / a.chunks, ch = was.pair - h * a.chunks, n_here = min(AD_HC, a.group - ch * AD_HC);
        const float l0 = __shfl_sync(0xffffffffu, l, 8 * t), l1 = __shfl_sync(0xffffffffu, l, 8 * t + 4);
        if (whole) {
            const float down = ad_pow2(max(v_exp, -116) - (AdStore<ST>::BF ? 0 : 10)), rest = ad_pow2(min(v_exp + 116, 0)); // 2^(v_exp - 10) in two factors
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                if (2 * t + b >= n_here) continue;
                const float inv = 1.f / (b ? l1 : l0);
                RT *out = (RT *)a.out.data + was.i * a.out.row_stride + (h * a.group + ch * AD_HC + 2 * t + b) * a.out.head_stride;
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    const float y0 = o[k][b] * inv * down * rest, y1 = o[k][2 + b] * inv * down * rest;
                    const int d = TL::v_dim(g, 2 * k);
                    if constexpr (std::is_same<RT, float>::value) *(float2 *)(out + d) = make_float2(y0, y1);
                    else if constexpr (std::is_same<RT, __half>::value) *(__half2 *)(out + d) = __floats2half2_rn(y0, y1);
                    else *(__nv_bfloat162 *)(out + d) = __floats2bfloat162_rn(y0, y1);
                }
            }
        } else {
            float *p = a.part + ((size_t)w * 2 + (first_seg ? 0 : 1)) * a.hc * (HD + 4);
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                if (2 * t + b >= n_here) continue;
                float *ph_ = p + (2 * t + b) * (HD + 4);
#pragma unroll
                for (int k = 0; k < KS; ++k) *(float2 *)(ph_ + TL::v_dim(g, 2 * k)) = make_float2(o[k][b], o[k][2 + b]);
            }
            if (t == 0 && g < n_here) *(float4 *)(p + g * (HD + 4) + HD) = make_float4(m, l, (float)v_exp, 0.f);
        }
        first_seg = false;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// Joins what the shares left of a (sequence, query head): grid (n_head, n_seq).  Sequences without rows get zeros.
template <typename RT, int HD>
__global__ void __launch_bounds__(AD_MERGE_THREADS) k_attn_decode_join(const AdArgs a, int p_exp) {
    constexpr int NW = AD_MERGE_THREADS / 32, EPL = HD >= 32 ? HD / 32 : 1;
    __shared__ float sm_m[NW], sm_l[NW], sm_o[NW][HD];
    __shared__ int sm_e[NW];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int hq = blockIdx.x, i = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    RT *out = (RT *)a.out.data + i * a.out.row_stride + hq * a.out.head_stride;
    const long long t0 = __ldcg(a.head + i), t1 = __ldcg(a.head + i + 1);
    const int n_tiles = (int)(t1 - t0);
    if (n_tiles == 0) {
        if (tid < HD) out[tid] = (RT)0.f;
        return;
    }
    const int pairs = a.c.n_kv_head * a.chunks, h = hq / a.group, hg = hq - h * a.group, pair = h * a.chunks + hg / AD_HC;
    const long long T = __ldcg(a.head + a.n_seq) * pairs, b0 = t0 * pairs + (long long)pair * n_tiles, b1 = b0 + n_tiles;
    const int W = ad_warps(a, T);
    const int w0 = (int)(((b0 + 1) * W - 1) / T), w1 = (int)((b1 * W - 1) / T); // shares that hold the first and the last tile
    if (w0 == w1) return;
    float m = -INFINITY, l = 0.f, o[EPL];
    int ex = -126;
#pragma unroll
    for (int e = 0; e < EPL; ++e) o[e] = 0.f;
    for (int w = w0 + warp; w <= w1; w += NW) {
        const int slot = w > w0 || ad_share(T, W, w) == b0 ? 0 : 1;
        const float *p = a.part + (((size_t)w * 2 + slot) * a.hc + hg % AD_HC) * (HD + 4);
        const float4 st = __ldcg((const float4 *)(p + HD));
        const float mn = fmaxf(m, st.x), ref = mn == -INFINITY ? 0.f : mn;
        const int ep = (int)st.z, en = max(ex, ep);
        const float f_old = ad_exp2(m - ref), f_new = ad_exp2(st.x - ref);
        const float g_old = f_old * ad_exp2((float)(ex - en)), g_new = f_new * ad_exp2((float)(ep - en));
        l = l * f_old + st.y * f_new;
        m = mn;
        ex = en;
#pragma unroll
        for (int e = 0; e < EPL; ++e)
            if (HD >= 32 || lane < HD) o[e] = o[e] * g_old + __ldcg(p + lane + 32 * e) * g_new;
    }
    if (lane == 0) { sm_m[warp] = m; sm_l[warp] = l; sm_e[warp] = ex; }
#pragma unroll
    for (int e = 0; e < EPL; ++e)
        if (HD >= 32 || lane < HD) sm_o[warp][lane + 32 * e] = o[e];
    __syncthreads();
    if (tid < HD) {
        float M = -INFINITY, L = 0.f, O = 0.f;
        int E = -126;
        for (int w = 0; w < NW; ++w) { M = fmaxf(M, sm_m[w]); E = max(E, sm_e[w]); }
        const float ref = M == -INFINITY ? 0.f : M;
        for (int w = 0; w < NW; ++w) {
            const float f = ad_exp2(sm_m[w] - ref);
            L += sm_l[w] * f;
            O += sm_o[w][tid] * f * ad_exp2((float)(sm_e[w] - E));
        }
        out[tid] = (RT)(O / L * ad_pow2(max(E, -116) - p_exp) * ad_pow2(min(E + 116, 0)));
    }
}

// ---- host --------------------------------------------------------------------------------------------------------
struct AdPlan { int chunks, hc, n_warps, min_tiles, blocks; int64_t bytes; };

AdPlan ad_plan(const mdi_kv_cache *c, int n_seq, int n_head, int max_len) {
    AdPlan p{};
    const int group = n_head / c->n_kv_head;
    p.chunks = (group + AD_HC - 1) / AD_HC;
    p.hc = std::min(group, AD_HC);
    const int64_t cap = (int64_t)c->pages_per_seq * c->page_tokens, len = max_len > 0 ? std::min<int64_t>(max_len, cap) : cap;
    const int64_t tiles = (int64_t)std::min(n_seq, AD_MAX_SEQ) * c->n_kv_head * p.chunks * ((len + 15) / 16);
    // a share of fewer tiles would leave more bytes of partial results than it reads
    p.min_tiles = 2 + p.hc / 2;
    const int resident = AD_SM * (op_scaled(c) ? 4 : 2) * AD_WARPS;
    p.n_warps = (int)std::max<int64_t>(1, std::min<int64_t>(resident, tiles / p.min_tiles));
    p.blocks = (p.n_warps + AD_WARPS - 1) / AD_WARPS;
    p.bytes = (AD_MAX_SEQ + 2) * 8 + (int64_t)p.n_warps * 2 * p.hc * (c->head_dim + 4) * 4;
    return p;
}

template <typename RT, int ST, int HD> cudaError_t ad_launch(const AdArgs &a, int blocks, cudaStream_t st) {
    constexpr size_t smem = ad_smem<ST, HD>();
    cudaError_t e = cudaFuncSetAttribute(k_attn_decode_op<RT, ST, HD>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    k_attn_decode_op<RT, ST, HD><<<blocks, AD_THREADS, smem, st>>>(a);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(a.n_head, a.n_seq);
    cfg.blockDim = dim3(AD_MERGE_THREADS);
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, k_attn_decode_join<RT, HD>, a, ST == AD_BF16 ? 0 : 10);
}
template <typename RT, int ST> cudaError_t ad_hd(const AdArgs &a, int blocks, cudaStream_t st) {
    switch (a.c.head_dim) {
        case 16: return ad_launch<RT, ST, 16>(a, blocks, st);
        case 32: return ad_launch<RT, ST, 32>(a, blocks, st);
        case 64: return ad_launch<RT, ST, 64>(a, blocks, st);
        default: return ad_launch<RT, ST, 128>(a, blocks, st);
    }
}
template <typename RT> cudaError_t ad_store(int kv_dtype, const AdArgs &a, int blocks, cudaStream_t st) {
    switch (kv_dtype) {
        case MDI_KV_I8: return ad_hd<RT, AD_I8>(a, blocks, st);
        case MDI_KV_E4M3: return ad_hd<RT, AD_E4M3>(a, blocks, st);
        case MDI_KV_F16: return ad_hd<RT, AD_F16>(a, blocks, st);
        default: return ad_hd<RT, AD_BF16>(a, blocks, st);
    }
}

int ad_check(const char *who, const mdi_kv_cache *cache, int n_seq, int n_head, int max_len) {
    const int rc = op_check_cache(who, cache);
    if (rc != MDI_OK) return rc;
    if (n_seq < 0) return op_fail(MDI_ERR_ARG, "%s: negative n_seq", who);
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
    return rc != MDI_OK ? rc : n_seq == 0 ? 0 : ad_plan(cache, n_seq, n_head, max_len).bytes;
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
    const AdPlan p = ad_plan(cache, std::max(n_seq, 1), n_head, max_len);
    if (n_seq > 0 && (!workspace_dev || workspace_bytes < p.bytes || ((uintptr_t)workspace_dev & 15)))
        return op_fail(MDI_ERR_ARG, "%s: needs a 16-byte aligned workspace of %lld bytes", who, (long long)p.bytes);
    if ((rc = op_check_ptrs(who, {{"pool_dev", cache->pool_dev, false}, {"scale_dev", cache->scale_dev, !op_scaled(cache)}, {"page_table_dev", cache->page_table_dev, false},
                                  {"q", q->data_dev, n_seq == 0}, {"out", out->data_dev, n_seq == 0}, {"slot_dev", slot_dev, true},
                                  {"len_dev", len_dev, false}, {"workspace_dev", workspace_dev, true}, {"status_dev", status_dev, true}})) != MDI_OK)
        return rc;
    for (int i0 = 0; i0 < n_seq; i0 += AD_MAX_SEQ) {
        AdArgs a{};
        a.c = op_cache(cache, slot_dev ? slot_dev + i0 : nullptr);
        a.q = op_rows(q); a.out = op_rows(out);
        const int64_t esize = q->dtype == MDI_DTYPE_F32 ? 4 : 2;
        a.q.data += i0 * a.q.row_stride * esize;
        a.out.data += i0 * a.out.row_stride * esize;
        a.len = len_dev + i0; a.status = status_dev;
        a.head = (long long *)workspace_dev;
        a.part = (float *)((char *)workspace_dev + (AD_MAX_SEQ + 2) * 8);
        a.n_seq = std::min(AD_MAX_SEQ, n_seq - i0); a.seq0 = i0;
        a.n_head = n_head; a.group = n_head / cache->n_kv_head;
        a.chunks = p.chunks; a.hc = p.hc; a.n_warps = p.n_warps; a.min_tiles = p.min_tiles;
        a.scale_log2e = scale * 1.4426950408889634f;
        cudaError_t e;
        OP_ROW_DISPATCH(q->dtype, (e = ad_store<RT>(cache->dtype, a, p.blocks, (cudaStream_t)stream)));
        if (e != cudaSuccess) return op_cuda(who, e);
    }
    return MDI_OK;
}
