// Attention of one new token per sequence over a paged key/value cache (mdi_attn_decode):
//     out[i][h] = sum_j softmax_j(scale * q[i][h] . K_j) V_j,   j < len[i],   K, V of key/value head h / group.
//
// Bound: the bytes of the cached rows.  What the layout is for:
//  * Work is cut into tiles of 32 cached rows, in units of 16 that never cross a page.  All tiles of all (sequence, key/value head,
//    chunk of up to 8 of its query heads) are laid end to end and dealt to the warps of the launch in equal contiguous
//    shares, so sequences of any mix of lengths keep every warp equally busy.  A (sequence, head) that a share boundary
//    cuts leaves partial results (maximum, sum, unnormalised output) in the workspace; a second, small kernel joins them in
//    a fixed order.  Nothing depends on timing.
//  * Where that leaves a warp next to nothing, a pair has a block, or a cluster of blocks, to itself instead (ad_plan).
//  * A warp streams its tiles through its own ring of shared memory with asynchronous copies of whole contiguous rows (a
//    unit's rows of one head are contiguous in its page).  16-byte chunks are stored swizzled, so that reading fragments has
//    no bank conflicts where rows have 128 bytes or more.  No barrier but the warp's own is needed.
//  * Products run on the tensor cores (mma.sync m16n8k16, fp32 accumulators), not for their rate but because one
//    instruction then serves the up to 8 query heads that share the row.  Scores: A = query (rows 0-7 the heads' high
//    parts, rows 8-15 their low parts), B = 8 cached rows; a lane then holds the scores of head lane / 4 for cached rows
//    2 (lane % 4), + 1, which is the layout that the B operand of the second product wants: A = V transposed (16 elements of
//    head_dim x 16 rows), B = weights.  Elements of head_dim and rows are assigned to fragment positions so that all copies
//    are wide and contiguous; both operands of a product use the same assignment.
//  * int8 keys with few heads each (ad_launch) are multiplied as they are (m16n8k32, exact 32-bit sums): a query is then an integer of 23
//    bits relative to the head's largest element, cut into three signed bytes, a row of A each (heads in rows 0-3, 4-7, 8-11).
//  * Other 8-bit elements become fp16 exactly in registers (int8: a byte under the exponent of 1024, minus 1152).  Scales stay
//    outside of the products: the key's multiplies the score, the value's the weight.
//  * Rounding: queries are used as two 16-bit planes (high + low, 16 to 22 bits together; scaled by a power of two per head where
//    the planes are fp16) or as those integers, weights as two planes, or as one fp16 where the output is 16 bits anyway (half a step of 2^-11 against
//    the output's own 2^-11 or 2^-8).  Weights refer to a running bound of score and value scale, so that fp16's range does not
//    matter.  Scores, weights' sums and outputs are fp32.
//
// Measured with both kernels, called from a host loop (bytes of cached rows over time; a plain copy moves 6.45 TB/s): 4 x 100003 e4m3
// rows, 40 heads on 8 of 128: 154 us, 5.5 TB/s; 64 x 640 int8 rows, 32 heads of 128, fp32: 75 us, 4.6 TB/s (some 10 of them to fill and
// empty the launch and to join); 32 ragged sequences up to 8192 bf16 rows: 31 us, 3.6 TB/s; 1000
// fp16 rows, 12 heads of 64: 11 us, most of it the host's (6 us on the device).
#include "ops_common.cuh"

#include <cuda_fp8.h>

#include <algorithm>
#include <type_traits>

namespace mdi {
namespace {

constexpr int AD_WARPS = 4;      // warps per block (they share nothing but the table of lengths)
constexpr int AD_THREADS = AD_WARPS * 32;
constexpr int AD_UNITS = 2;      // 16-row units per tile: one softmax step serves 32 rows.  16 rows: 86 instead of 78 us (64 x 640 int8 rows, 32 heads of 128), 39 instead of 32 us (32 ragged sequences up to 8192 bf16 rows, 32 heads on 8)
constexpr int AD_STAGES = 2;     // tiles in a warp's ring.  3 leave room for fewer blocks: 4 to 9% slower
constexpr int AD_MAX_BLOCKS = 4; // resident blocks per SM
constexpr int AD_MAX_SEQ = 256;  // sequences per launch (their table shares shared memory with the rings of 4 blocks per SM)
constexpr int AD_HC = 8;         // query heads per chunk
constexpr int AD_SM = 148;
constexpr int AD_TURN = 2;       // see ad_places (1, 2, 4: within 2%; 0: 44 instead of 32 us for the ragged sequences above)
constexpr float AD_SLACK = 4.f;  // a maximum may be exceeded by 2^4 before what has been summed is rescaled
constexpr int AD_JOIN_THREADS = 128;

struct AdArgs {
    OpCache c;
    OpRows q, out;
    const int *len;
    int *status;
    float *part;      // workspace: [warps][pair from an earlier share | pair that goes on in a later one][hc][HD + 4]: output (not yet divided), what its weights refer to, their sum
    int n_seq, seq0;  // sequences of this launch, first one's number
    int n_head, group, chunks, hc, n_warps, min_tiles;
    int whole; // blocks that a pair has to itself (a cluster), 0: tiles are dealt to warps; see ad_plan
    float scale_log2e;
};

enum { AD_I8, AD_E4M3, AD_F16, AD_BF16 };
template <int ST> struct AdStore {
    static constexpr int SIZE = ST <= AD_E4M3 ? 1 : 2;
    static constexpr bool SCALED = SIZE == 1, BF = ST == AD_BF16;
};

__device__ __forceinline__ void ad_mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, std::false_type) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ad_mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, std::true_type) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// d += a (b + c), rounded to nearest
template <typename BF> __device__ __forceinline__ void ad_mma_add(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, uint32_t c0, uint32_t c1, BF) {
    float f[4] = {0.f, 0.f, 0.f, 0.f};
    ad_mma(f, a, c0, c1, BF());
    ad_mma(f, a, b0, b1, BF());
#pragma unroll
    for (int e = 0; e < 4; ++e) d[e] += f[e];
}
__device__ __forceinline__ void ad_mma(int (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float ad_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float ad_log2(float x) {
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
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
        uint32_t r; // (the intrinsic works on 16-bit pieces, which cost a permutation each to take apart and to put together)
        if constexpr (UPPER) asm("{\n .reg .b16 lo, hi;\n mov.b32 {lo, hi}, %1;\n cvt.rn.f16x2.e4m3x2 %0, hi;\n}\n" : "=r"(r) : "r"(w));
        else asm("{\n .reg .b16 lo, hi;\n mov.b32 {lo, hi}, %1;\n cvt.rn.f16x2.e4m3x2 %0, lo;\n}\n" : "=r"(r) : "r"(w));
        return r;
    }
}
template <int ST> __device__ __forceinline__ uint32_t ad_bias(uint32_t w) { return ST == AD_I8 ? w ^ 0x80808080u : w; }

__device__ __forceinline__ void ad_cluster_meet() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ float ad_remote(uint32_t addr, uint32_t rank) { // a float of block `rank` of the cluster
    float x;
    asm volatile("{\n .reg .b32 a;\n mapa.shared::cluster.u32 a, %1, %2;\n ld.shared::cluster.f32 %0, [a];\n}\n" : "=f"(x) : "r"(addr), "r"(rank) : "memory");
    return x;
}
// 16 bytes from global to shared memory, zeros where !ok
__device__ __forceinline__ void ad_copy16(uint32_t dst, const unsigned char *src, bool ok) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0) : "memory");
}
__device__ __forceinline__ void ad_copy4(uint32_t dst, const float *src, bool ok) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(ok ? 4 : 0) : "memory");
}
template <int BYTES> __device__ __forceinline__ void ad_read(uint32_t (&w)[(BYTES + 3) / 4], const unsigned char *p) {
    if constexpr (BYTES == 16) { const uint4 v = *(const uint4 *)p; w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w; }
    else if constexpr (BYTES == 8) { const uint2 v = *(const uint2 *)p; w[0] = v.x; w[1] = v.y; }
    else if constexpr (BYTES == 4) w[0] = *(const uint32_t *)p;
    else w[0] = *(const unsigned short *)p;
}
__device__ __forceinline__ float2 ad_read2(const unsigned char *p) { return *(const float2 *)p; }
__device__ __forceinline__ int ad_read1(const unsigned char *p) { return *(const int *)p; }

// A unit in shared memory: 16 rows of keys, 16 rows of values, RB bytes each, 16-byte chunk c of row r at chunk c ^ swizzle(r).
// As fragments, g = lane / 4, t = lane % 4: of the keys a lane reads rows g and g + 8, a quarter of each (KN pieces of KC bytes);
// of the values rows 2t, 2t + 1, 2t + 8, 2t + 9, an eighth of each (VN pieces of VC bytes).
template <int ST, int HD> struct AdTile {
    static constexpr int SZ = AdStore<ST>::SIZE, RB = HD * SZ;
    static constexpr int KB = RB / 4, KC = KB < 16 ? KB : 16, KN = KB / KC;
    static constexpr int VB = RB / 8, VC = VB < 16 ? VB : 16, VN = VB / VC;
    static constexpr int U = AD_UNITS, ROWS = 16 * U;
    static constexpr int K_BYTES = 16 * RB, UNIT = 2 * K_BYTES;
    static constexpr int SCALES = U * UNIT, LIVE = SCALES + (SZ == 1 ? U * 128 : 0); // per unit 16 + 16 scales, then the number of rows
    static constexpr int STAGE = LIVE + 16, STAGES = AD_STAGES;
    static constexpr int BLOCK_SMEM = AD_WARPS * STAGES * STAGE + (AD_MAX_SEQ + 1) * 8 + AD_MAX_SEQ * 4;
    static constexpr int FIT = (227 * 1024) / (BLOCK_SMEM + 1024), BLOCKS = FIT < AD_MAX_BLOCKS ? FIT : AD_MAX_BLOCKS; // resident blocks per SM
    static __device__ __forceinline__ int at(int row, int byte) {
        const int sw = RB >= 128 ? row & 7 : RB == 64 ? (row >> 1) & 3 : 0;
        return row * RB + ((byte & ~15) ^ (sw << 4)) + (byte & 15);
    }
    static __device__ __forceinline__ int k_byte(int t, int c) { return RB >= 128 ? (2 * t + (c & 1) + 8 * (c >> 1)) * 16 : t * KC; } // lane's piece c of a row of keys
    static __device__ __forceinline__ int v_byte(int g, int c) { return g * VC + c * 128; }
    static __device__ __forceinline__ int k_dim(int t, int s) { const int b = 4 * s * SZ; return (k_byte(t, b / KC) + b % KC) / SZ; } // first of a lane's 4 elements of k-step s
    static __device__ __forceinline__ int v_dim(int g, int j) { const int b = j * SZ; return (v_byte(g, b / VC) + b % VC) / SZ; }     // a lane's j-th element
};

__device__ __forceinline__ int ad_len(const AdArgs &a, int i, int *status) {
    const int n = a.len[i], slot = a.c.slot ? a.c.slot[i] : a.seq0 + i;
    if ((unsigned)slot >= (unsigned)a.c.n_slots || n < 0) { op_status(status, MDI_STATUS_RANGE); return 0; }
    if (n > a.c.capacity) { op_status(status, MDI_STATUS_RANGE); return (int)a.c.capacity; }
    return n;
}

// Places in the line of tiles.  Every pair is followed by AD_TURN places without a tile, which stand for what it costs a warp to
// finish a pair and begin the next: without them, shares full of very short sequences take far longer than the others.
__device__ __forceinline__ int ad_places(int n_tiles) { return n_tiles > 0 ? n_tiles + AD_TURN : 0; }

template <int ROWS> __device__ __forceinline__ int ad_tiles(int len) { return (int)(((unsigned)len + ROWS - 1) / ROWS); }

// Where in the line: sequence, (head, chunk) pair within it, tile within the pair
template <int ROWS> struct AdCursor {
    int i, pair, tile, n_tiles, len;
    long long at; // its place
    __device__ __forceinline__ void enter(const int *s_len, int seq) { i = seq; len = s_len[seq]; n_tiles = ad_tiles<ROWS>(len); }
    // the first tile at or behind place `first`
    __device__ __forceinline__ void seek(const long long *pref, const int *s_len, int n_seq, int pairs, long long first) {
        int lo = 0, hi = n_seq - 1; // last sequence that begins at or before it
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (pref[mid] * pairs <= first) lo = mid; else hi = mid - 1;
        }
        enter(s_len, lo);
        const long long in = first - pref[lo] * pairs;
        const int per = ad_places(n_tiles);
        pair = in <= 0x7fffffff ? (int)in / per : (int)(in / per); // (a 32-bit division where it will do)
        tile = (int)(in - (long long)pair * per);
        at = first;
        if (tile >= n_tiles) {
            at += per - tile;
            next_pair(s_len, n_seq, pairs);
        }
    }
    __device__ __forceinline__ void next_pair(const int *s_len, int n_seq, int pairs) {
        tile = 0;
        if (++pair == pairs) {
            pair = 0;
            do ++i; while (i < n_seq && s_len[i] == 0);
            if (i < n_seq) enter(s_len, i);
        }
    }
    // this warp's part of a pair that has `warps` warps to itself
    __device__ __forceinline__ long long part(int seq, int in_seq, int rows, int warp, int warps) {
        i = seq; pair = in_seq; len = rows; n_tiles = ad_tiles<ROWS>(rows);
        tile = (int)((long long)n_tiles * warp / warps);
        at = tile;
        return (long long)n_tiles * (warp + 1) / warps;
    }
    // true: the next tile belongs to another pair
    __device__ __forceinline__ bool advance(const int *s_len, int n_seq, int pairs, bool whole) {
        ++at;
        if (++tile < n_tiles || whole) return false;
        at += AD_TURN;
        next_pair(s_len, n_seq, pairs);
        return true;
    }
};

// share of warp w: places [T w / W, T (w + 1) / W)
__device__ __forceinline__ long long ad_share(long long T, int W, int w) { return T * w / W; }
__device__ __forceinline__ int ad_warps(const AdArgs &a, long long T) {
    const long long w = T / a.min_tiles;
    return (int)(w < 1 ? 1 : w < a.n_warps ? w : a.n_warps);
}

// QI: int8 keys as they are (see the top of the file)
template <typename RT, int ST, int HD, bool QI>
__global__ void __launch_bounds__(AD_THREADS, AdTile<ST, HD>::BLOCKS) k_attn_decode_op(const AdArgs a) {
    using TL = AdTile<ST, HD>;
    using BF = std::integral_constant<bool, AdStore<ST>::BF>;
    constexpr bool SCALED = AdStore<ST>::SCALED;
    constexpr int U = TL::U, STAGES = TL::STAGES;
    constexpr int KS = HD / 16;                       // k-steps of the scores, m-tiles of the output
    constexpr float UP = AdStore<ST>::BF ? 0.f : 10.f; // weights times value scales stay below 2^(UP + AD_SLACK): inside fp16's range, far from its end
    constexpr bool PLO = AdStore<ST>::BF || std::is_same<RT, float>::value; // low parts of the weights: see the top of the file
    // fp32 outputs: the matrix instruction cuts off what it adds to a larger accumulator, always towards zero, so 16 rows at a time are
    // multiplied into a fresh one and added to the output with rounding (640 int8 rows: relative error 6.7e-7 instead of 1.3e-6 for 75.2
    // instead of 73.6 us)
    constexpr bool RN = std::is_same<RT, float>::value;
    extern __shared__ __align__(16) unsigned char ad_raw[];
    long long *s_pref = (long long *)(ad_raw + AD_WARPS * STAGES * TL::STAGE);
    int *s_len = (int *)(s_pref + AD_MAX_SEQ + 1);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    // ---- lengths, places before each sequence (every block for itself)
    if (!a.whole) {
        __shared__ long long s_sum[AD_WARPS];
        long long run = 0;
        for (int base = 0; base < a.n_seq; base += AD_THREADS) {
            const int i = base + tid;
            const int n = i < a.n_seq ? ad_len(a, i, blockIdx.x == 0 ? a.status : nullptr) : 0;
            const long long mine = ad_places(ad_tiles<TL::ROWS>(n));
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
            }
            __syncthreads();
        }
        if (tid == 0) s_pref[a.n_seq] = run;
        __syncthreads();
    }
    const int pairs = a.c.n_kv_head * a.chunks;
    const int w = blockIdx.x * AD_WARPS + warp;
    long long first, last;
    AdCursor<TL::ROWS> cur, nxt; // consumer, producer
    if (a.whole) {
        const int mine = blockIdx.x / a.whole, rank = blockIdx.x - mine * a.whole, i = mine / pairs, in = mine - i * pairs;
        last = cur.part(i, in, ad_len(a, i, in == 0 && rank == 0 && tid == 0 ? a.status : nullptr), rank * AD_WARPS + warp, a.whole * AD_WARPS);
        first = cur.at;
    } else {
        const long long T = s_pref[a.n_seq] * pairs;
        const int W = ad_warps(a, T);
        if (T == 0 || w >= W) return;
        first = ad_share(T, W, w);
        last = ad_share(T, W, w + 1);
        cur.seek(s_pref, s_len, a.n_seq, pairs, first);
        if (cur.at >= last) return;
    }
    nxt = cur;
    int batch_i = -1, batch_tile = 0, batch_page = -1, page_slot = 0;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(ad_raw) + warp * STAGES * TL::STAGE;
    const long long head_rows = (long long)a.c.n_kv_head << a.c.page_shift; // rows of one half of a page

    // The next tile into stage `s`.  The lanes hold the page numbers of the next 32 tiles; the rows of a page that does not exist
    // count as behind the end.
    auto load = [&](int s) {
        if (nxt.at < last) {
            if (batch_i != nxt.i || nxt.tile < batch_tile || nxt.tile == 0 || nxt.tile >= batch_tile + 32 / U) {
                if (batch_i >= 0 && nxt.tile == 0 && lane < a.hc) { // a new pair's queries, before they are wanted
                    const int qh = nxt.pair / a.chunks * a.group + nxt.pair % a.chunks * AD_HC + lane;
                    if (nxt.pair % a.chunks * AD_HC + lane < a.group) {
                        const unsigned char *q = a.q.data + (nxt.i * a.q.row_stride + qh * a.q.head_stride) * (long long)sizeof(RT);
#pragma unroll
                        for (int b = 0; b < HD * (int)sizeof(RT); b += 128) asm volatile("prefetch.global.L1 [%0];" ::"l"(q + b));
                    }
                }
                batch_i = nxt.i;
                batch_tile = nxt.tile;
                page_slot = a.c.slot ? a.c.slot[nxt.i] : a.seq0 + nxt.i;
                batch_page = -1;
                const unsigned row = (unsigned)(batch_tile * U + lane) << 4; // (may pass 2^31 next to the largest length)
                if (row < (unsigned)nxt.len) {
                    batch_page = __ldg(a.c.table + (long long)page_slot * a.c.table_stride + (row >> a.c.page_shift));
                    if ((unsigned)batch_page >= (unsigned)a.c.n_pages) { op_status(a.status, MDI_STATUS_PAGE); batch_page = -1; }
                }
            }
            const int h = a.chunks == 1 ? nxt.pair : nxt.pair / a.chunks;
            const uint32_t st = ring + s * TL::STAGE;
            long long kr = 0; // row of the pool
            int page = -1;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const unsigned row0 = (unsigned)(nxt.tile * U + u) << 4;
                if (u == 0 || a.c.page_shift == 4) {
                    page = __shfl_sync(0xffffffffu, batch_page, (nxt.tile - batch_tile) * U + u);
                    kr = page < 0 ? 0 : ((((long long)page * 2) * a.c.n_kv_head + h) << a.c.page_shift) + (int)(row0 & ((1u << a.c.page_shift) - 1));
                } else kr += page < 0 ? 0 : 16;
                const int rows = page < 0 ? 0 : min(16, (int)((unsigned)nxt.len - row0));
                const unsigned char *kp = a.c.pool + kr * TL::RB + lane * 16, *vp = kp + head_rows * TL::RB;
                const uint32_t sk = st + u * TL::UNIT;
                constexpr int COPIES = TL::K_BYTES / 512; // of 32 chunks; rows of 16 bytes: half of one
                if (COPIES > 0 || lane < 16) {
#pragma unroll
                    for (int i = 0; i < (COPIES > 0 ? COPIES : 1); ++i) {
                        const int row = (i * 512 + lane * 16) / TL::RB, dst = TL::at(row, (i * 512 + lane * 16) % TL::RB);
                        ad_copy16(sk + dst, kp + i * 512, row < rows);
                        ad_copy16(sk + TL::K_BYTES + dst, vp + i * 512, row < rows);
                    }
                }
                if (SCALED) { // lanes 0-15 the keys' scales, 16-31 the values'
                    const int row = lane & 15;
                    ad_copy4(st + TL::SCALES + u * 128 + lane * 4, a.c.scale + kr + (lane >> 4) * head_rows + row, row < rows);
                }
                if (lane == 0) asm volatile("st.shared.s32 [%0], %1;" ::"r"(st + TL::LIVE + u * 4), "r"(rows) : "memory");
            }
            nxt.advance(s_len, a.n_seq, pairs, a.whole);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };

#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) load(s);

    uint32_t qa[QI ? KS / 2 : KS][4]; // queries as fragments
    float o[KS][4], m = -INFINITY, l = 0.f, q_up = 1.f; // m: what weights refer to, 2^(score - m); l: their sum
    bool fresh = true;
    int stage = 0;
    while (cur.at < last) {
        if (fresh) { // a new (sequence, head, chunk): its queries, scaled into log2 units, as fragments
            fresh = false;
            const int h = cur.pair / a.chunks, ch = cur.pair - h * a.chunks;
            const int qg = QI ? g & 3 : g; // head of the group
            const int qh = h * a.group + ch * AD_HC + qg;
            const bool there = ch * AD_HC + qg < a.group;
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
            if (!AdStore<ST>::BF) { // fp16 planes: the largest element to [2^12, 2^13), so that low parts stay normal numbers
                big = max(big, __shfl_xor_sync(0xffffffffu, big, 1));
                big = max(big, __shfl_xor_sync(0xffffffffu, big, 2));
                if (big != 0 && big < 0x7f800000u) { // (QI: to [2^21, 2^22))
                    const int e = min(max((int)(big >> 23) - (QI ? 148 : 139), -126), 126);
                    q_up = ad_pow2(e);
                    q_down = ad_pow2(-e);
                } else if (QI && big != 0) {
                    q_up = __uint_as_float(0x7fc00000u); // a query that is not finite: NaN
                    q_down = 0.f;
                }
            }
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                if constexpr (QI) {
                    uint32_t v[4], w[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int i = __float2int_rn(f[s][e] * q_down);
                        v[e] = (uint32_t)(g < 4 ? (i + 0x8080) >> 16 : (i + 0x80) >> 8); // (its low byte counts, signed)
                        w[e] = (uint32_t)i;
                    }
                    qa[s / 2][s % 2 * 2] = __byte_perm(__byte_perm(v[0], v[1], 0x0040), __byte_perm(v[2], v[3], 0x0040), 0x5410);
                    qa[s / 2][s % 2 * 2 + 1] = g < 4 ? __byte_perm(__byte_perm(w[0], w[1], 0x0040), __byte_perm(w[2], w[3], 0x0040), 0x5410) : 0u;
                } else {
                    ad_split(f[s][0] * q_down, f[s][1] * q_down, qa[s][0], qa[s][1], BF());
                    ad_split(f[s][2] * q_down, f[s][3] * q_down, qa[s][2], qa[s][3], BF());
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) o[s][e] = 0.f;
            }
            m = -INFINITY;
            l = 0.f;
        }
        asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
        __syncwarp();
        load(stage == 0 ? STAGES - 1 : stage - 1); // the stage that the previous tile used
        const unsigned char *st = ad_raw + (warp * STAGES + stage) * TL::STAGE;
        stage = stage == STAGES - 1 ? 0 : stage + 1;

        // ---- scores: s[2 u + r] are rows 16 u + 8 r + 2t, + 1 for head g (high part of the query, then low part)
        std::conditional_t<QI, int, float> s[2 * U][4];
#pragma unroll
        for (int r = 0; r < 2 * U; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[r][e] = 0;
#pragma unroll
        for (int c = 0; c < TL::KN; ++c) {
            constexpr int KPC = TL::KC * 4 / (TL::SZ * 16); // k-steps in a chunk
            uint32_t kw[2 * U][(TL::KC + 3) / 4];
#pragma unroll
            for (int r = 0; r < 2 * U; ++r) ad_read<TL::KC>(kw[r], st + r / 2 * TL::UNIT + r % 2 * 8 * TL::RB + TL::at(g, TL::k_byte(t, c)));
            if constexpr (QI) {
#pragma unroll
                for (int k = 0; k < KPC; k += 2)
#pragma unroll
                    for (int r = 0; r < 2 * U; ++r) ad_mma(s[r], qa[(c * KPC + k) / 2], kw[r][k], kw[r][k + 1]);
                continue;
            } else
#pragma unroll
            for (int k = 0; k < KPC; ++k)
#pragma unroll
                for (int r = 0; r < 2 * U; ++r) {
                    uint32_t b0, b1;
                    if constexpr (TL::SZ == 1) {
                        const uint32_t w = ad_bias<ST>(kw[r][k]);
                        b0 = ad_wide<ST, 0>(w);
                        b1 = ad_wide<ST, 1>(w);
                    } else {
                        b0 = kw[r][2 * k];
                        b1 = kw[r][2 * k + 1];
                    }
                    ad_mma(s[r], qa[c * KPC + k], b0, b1, BF());
                }
        }
        float x[4 * U], vs[4 * U]; // scores (times q_up: in log2 units), scales of the values; [4 u + 2 r + b] is row 16 u + 8 r + 2t + b
#pragma unroll
        for (int r = 0; r < 2 * U; ++r) {
            float2 ks = make_float2(1.f, 1.f), v2 = ks;
            if (SCALED) {
                const unsigned char *sc = st + TL::SCALES + r / 2 * 128 + (8 * (r % 2) + 2 * t) * 4;
                ks = ad_read2(sc);
                v2 = ad_read2(sc + 64);
            }
            vs[2 * r] = v2.x;
            vs[2 * r + 1] = v2.y;
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                if constexpr (QI) { // rows 0-3 hold the heads' highest bytes, 4-7 the middle, 8-11 the lowest
                    const int middle = __shfl_xor_sync(0xffffffffu, s[r][b], 16);
                    const float sum = fmaf((float)s[r][b], 65536.f, fmaf((float)middle, 256.f, (float)s[r][2 + b]));
                    x[2 * r + b] = g < 4 ? sum * (b ? ks.y : ks.x) : 0.f;
                } else {
                    float sum = s[r][b] + s[r][2 + b];
                    // a 16-bit key may be infinite: the low part of the query, of either sign or zero, has no say then
                    if (!SCALED && fabsf(s[r][b]) == INFINITY) sum = s[r][b];
                    x[2 * r + b] = SCALED ? sum * (b ? ks.y : ks.x) : sum;
                }
            }
        }
        // ---- rows behind the end, or of a page that does not exist
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int live = ad_read1(st + TL::LIVE + u * 4);
            if (live < 16) {
#pragma unroll
                for (int r = 0; r < 2; ++r)
#pragma unroll
                    for (int b = 0; b < 2; ++b)
                        if (8 * r + 2 * t + b >= live) { x[4 * u + 2 * r + b] = -INFINITY; vs[4 * u + 2 * r + b] = 0.f; }
            }
        }
        // ---- what the weights refer to: the largest score, plus the exponent of the largest value scale (weight times scale is
        // what has to fit fp16; numerator and denominator share the reference); it moves only when exceeded by the slack.  The bounds on
        // the exponent keep the weights' sum finite for 2^31 rows (weights up to 2^(80 + 14)) and the largest weight above 2^-114.
        float top = x[0], big = vs[0];
#pragma unroll
        for (int i = 1; i < 4 * U; ++i) { top = fmaxf(top, x[i]); big = fmaxf(big, vs[i]); }
        top = top * q_up - UP;
        if (SCALED) top += ad_log2(fminf(fmaxf(big, 0x1p-80f), 0x1p119f));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const bool rise = top > m + AD_SLACK || (m == -INFINITY && top > -INFINITY);
        if (__any_sync(0xffffffffu, rise)) {
            const float f = rise ? (m == -INFINITY ? 0.f : ad_exp2(m - top)) : 1.f;
            l *= f;
            if (rise) m = top;
            const float f0 = __shfl_sync(0xffffffffu, f, 8 * t), f1 = __shfl_sync(0xffffffffu, f, 8 * t + 4); // heads 2t, 2t + 1
#pragma unroll
            for (int k = 0; k < KS; ++k) { o[k][0] *= f0; o[k][1] *= f1; o[k][2] *= f0; o[k][3] *= f1; }
        }
        const float ref = m == -INFINITY ? 0.f : m;
        uint32_t ph[2 * U], pl[2 * U];
#pragma unroll
        for (int r = 0; r < 2 * U; ++r) {
            float p0 = ad_exp2(fmaf(x[2 * r], q_up, -ref)), p1 = ad_exp2(fmaf(x[2 * r + 1], q_up, -ref));
            l += p0 + p1;
            if (SCALED) { p0 *= vs[2 * r]; p1 *= vs[2 * r + 1]; }
            ad_split(p0, p1, ph[r], pl[r], BF());
        }
        // ---- values
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int c = 0; c < TL::VN; ++c) {
                constexpr int WORDS = (TL::VC + 3) / 4;
                uint32_t vw[4][WORDS];
#pragma unroll
                for (int r = 0; r < 4; ++r) ad_read<TL::VC>(vw[r], st + u * TL::UNIT + TL::K_BYTES + r / 2 * 8 * TL::RB + TL::at(2 * t + r % 2, TL::v_byte(g, c)));
#pragma unroll
                for (int i = 0; i < WORDS; ++i) {
                    if constexpr (TL::SZ == 1) {
                        const uint32_t x0 = ad_bias<ST>(vw[0][i]), x1 = ad_bias<ST>(vw[1][i]), x2 = ad_bias<ST>(vw[2][i]), x3 = ad_bias<ST>(vw[3][i]);
                        const int k = (c * WORDS + i) * 2; // a word holds the elements of two m-tiles
                        uint32_t av[4], aw[4];
                        uint32_t y = __byte_perm(x0, x1, 0x5140), z = __byte_perm(x2, x3, 0x5140);
                        av[0] = ad_wide<ST, 0>(y); av[1] = ad_wide<ST, 1>(y); av[2] = ad_wide<ST, 0>(z); av[3] = ad_wide<ST, 1>(z);
                        if constexpr (!RN) ad_mma(o[k], av, ph[2 * u], ph[2 * u + 1], BF());
                        if constexpr (TL::VC >= 4) {
                            y = __byte_perm(x0, x1, 0x7362); z = __byte_perm(x2, x3, 0x7362);
                            aw[0] = ad_wide<ST, 0>(y); aw[1] = ad_wide<ST, 1>(y); aw[2] = ad_wide<ST, 0>(z); aw[3] = ad_wide<ST, 1>(z);
                            if constexpr (!RN) ad_mma(o[k + 1], aw, ph[2 * u], ph[2 * u + 1], BF());
                        }
                        if constexpr (RN) {
                            ad_mma_add(o[k], av, ph[2 * u], ph[2 * u + 1], pl[2 * u], pl[2 * u + 1], BF());
                            if constexpr (TL::VC >= 4) ad_mma_add(o[k + 1], aw, ph[2 * u], ph[2 * u + 1], pl[2 * u], pl[2 * u + 1], BF());
                        } else if constexpr (PLO) {
                            ad_mma(o[k], av, pl[2 * u], pl[2 * u + 1], BF());
                            if constexpr (TL::VC >= 4) ad_mma(o[k + 1], aw, pl[2 * u], pl[2 * u + 1], BF());
                        }
                    } else {
                        const int k = c * WORDS + i;
                        uint32_t av[4];
                        av[0] = __byte_perm(vw[0][i], vw[1][i], 0x5410);
                        av[1] = __byte_perm(vw[0][i], vw[1][i], 0x7632);
                        av[2] = __byte_perm(vw[2][i], vw[3][i], 0x5410);
                        av[3] = __byte_perm(vw[2][i], vw[3][i], 0x7632);
                        if constexpr (RN) {
                            ad_mma_add(o[k], av, ph[2 * u], ph[2 * u + 1], pl[2 * u], pl[2 * u + 1], BF());
                        } else {
                            ad_mma(o[k], av, ph[2 * u], ph[2 * u + 1], BF());
                            if constexpr (PLO) ad_mma(o[k], av, pl[2 * u], pl[2 * u + 1], BF());
                        }
                    }
                }
            }
        // ---- the end of this pair, or of this warp's share of it
        const AdCursor<TL::ROWS> was = cur;
        const bool turn = cur.advance(s_len, a.n_seq, pairs, a.whole);
        if (!turn && cur.at < last) continue;
        l += __shfl_xor_sync(0xffffffffu, l, 1);
        l += __shfl_xor_sync(0xffffffffu, l, 2);
        if (a.whole) break;
        fresh = true;
        const bool from_start = was.at - was.tile >= first, whole = turn && from_start; // a pair that began in an earlier share has its tile 0 there
        const int h = was.pair / a.chunks, ch = was.pair - h * a.chunks, n_here = min(AD_HC, a.group - ch * AD_HC);
        const float l0 = __shfl_sync(0xffffffffu, l, 8 * t), l1 = __shfl_sync(0xffffffffu, l, 8 * t + 4);
        if (whole) {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                if (2 * t + b >= n_here) continue;
                const float sum = b ? l1 : l0, inv = sum == 0.f ? 0.f : 1.f / sum; // 0: no row is left, or all scores are -inf
                RT *out = (RT *)a.out.data + was.i * a.out.row_stride + (h * a.group + ch * AD_HC + 2 * t + b) * a.out.head_stride;
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    const float y0 = o[k][b] * inv, y1 = o[k][2 + b] * inv;
                    const int d = TL::v_dim(g, 2 * k);
                    if constexpr (std::is_same<RT, float>::value) *(float2 *)(out + d) = make_float2(y0, y1);
                    else if constexpr (std::is_same<RT, __half>::value) *(__half2 *)(out + d) = __floats2half2_rn(y0, y1);
                    else *(__nv_bfloat162 *)(out + d) = __floats2bfloat162_rn(y0, y1);
                }
            }
        } else {
            float *p = a.part + ((size_t)w * 2 + (from_start ? 1 : 0)) * a.hc * (HD + 4);
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                if (2 * t + b >= n_here) continue;
                float *ph_ = p + (2 * t + b) * (HD + 4);
#pragma unroll
                for (int k = 0; k < KS; ++k) *(float2 *)(ph_ + TL::v_dim(g, 2 * k)) = make_float2(o[k][b], o[k][2 + b]);
            }
            if (t == 0 && g < n_here) *(float4 *)(p + g * (HD + 4) + HD) = make_float4(m, l, 0.f, 0.f);
        }
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    if (!a.whole) return;
    // ---- a pair to itself: the warps' parts meet in shared memory (where the rings were) and are joined in their order; those of a
    // cluster's blocks after that
    float (*s_o)[AD_HC][HD + 4] = reinterpret_cast<float (*)[AD_HC][HD + 4]>(ad_raw); // [warp, then the block][head]: output, what its weights refer to, their sum
    static_assert((AD_WARPS + 1) * AD_HC * (HD + 4) * 4 <= AD_WARPS * STAGES * TL::STAGE, "the rings hold the parts");
    const int mine = blockIdx.x / a.whole, rank = blockIdx.x - mine * a.whole, seq = mine / pairs, in = mine - seq * pairs;
    const int h = in / a.chunks, ch = in - h * a.chunks, n_here = min(AD_HC, a.group - ch * AD_HC);
    const bool some = first < last;
    __syncthreads();
    if (some) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int k = 0; k < KS; ++k) *(float2 *)&s_o[warp][2 * t + b][TL::v_dim(g, 2 * k)] = make_float2(o[k][b], o[k][2 + b]);
    }
    if (t == 0) *(float2 *)&s_o[warp][g][HD] = some ? make_float2(m, l) : make_float2(-INFINITY, 0.f);
    __syncthreads();
    // joins `n` parts, the x-th of which is at part(x, element); -> output (not divided), reference, sum
    auto join = [&](int n, auto part, float (&y)[(HD + 31) / 32], float &top, float &sum) {
        top = -INFINITY;
        sum = 0.f;
        for (int x = 0; x < n; ++x) top = fmaxf(top, part(x, HD));
        const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int e = 0; e < (HD + 31) / 32; ++e) y[e] = 0.f;
        for (int x = 0; x < n; ++x) {
            const float f = ad_exp2(part(x, HD) - ref), s = part(x, HD + 1);
            if (s == 0.f) continue; // (nothing was seen, and no output written)
            sum += s * f;
#pragma unroll
            for (int e = 0; e < (HD + 31) / 32; ++e)
                if (HD >= 32 || lane < HD) y[e] += part(x, lane + 32 * e) * f;
        }
    };
    auto store = [&](int q, const float (&y)[(HD + 31) / 32], float sum) {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        RT *out = (RT *)a.out.data + seq * a.out.row_stride + (h * a.group + ch * AD_HC + q) * a.out.head_stride;
#pragma unroll
        for (int e = 0; e < (HD + 31) / 32; ++e)
            if (HD >= 32 || lane < HD) out[lane + 32 * e] = (RT)(y[e] * inv);
    };
    float y[(HD + 31) / 32], top, sum;
    for (int q = warp; q < n_here; q += AD_WARPS) {
        join(AD_WARPS, [&](int x, int e) { return s_o[x][q][e]; }, y, top, sum);
        if (a.whole == 1) { store(q, y, sum); continue; }
#pragma unroll
        for (int e = 0; e < (HD + 31) / 32; ++e)
            if (HD >= 32 || lane < HD) s_o[AD_WARPS][q][lane + 32 * e] = y[e];
        if (lane == 0) *(float2 *)&s_o[AD_WARPS][q][HD] = make_float2(top, sum);
    }
    if (a.whole == 1) return;
    ad_cluster_meet();
    const uint32_t there = (uint32_t)__cvta_generic_to_shared(&s_o[AD_WARPS][0][0]);
    for (int q = rank * AD_WARPS + warp; q < n_here; q += a.whole * AD_WARPS) { // the heads are shared out among all warps of the cluster
        join(a.whole, [&](int x, int e) { return ad_remote(there + (q * (HD + 4) + e) * 4, x); }, y, top, sum);
        store(q, y, sum);
    }
    ad_cluster_meet(); // nothing is read from a block that has gone
}

// Joins what the shares left of a (sequence, query head); NW warps per head, grid (heads / (4 / NW), n_seq).  Sequences without
// rows get zeros.  What to join follows from the lengths alone, so that is worked out before waiting for the main kernel.
template <typename RT, int HD, int NW>
__global__ void __launch_bounds__(AD_JOIN_THREADS) k_attn_decode_join(const AdArgs a) {
    constexpr int EPL = HD >= 32 ? HD / 32 : 1, AHEAD = 8;
    __shared__ float sm_m[4], sm_l[4], sm_o[4][HD];
    __shared__ long long sm_before[4], sm_total[4];
    const int i = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int hq = blockIdx.x * (4 / NW) + warp / NW, part_no = warp % NW;
    long long before = 0, total = 0;
    for (int j = tid; j < a.n_seq; j += AD_JOIN_THREADS) {
        const long long n = ad_places(ad_tiles<16 * AD_UNITS>(ad_len(a, j, nullptr)));
        total += n;
        if (j < i) before += n;
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        before += __shfl_xor_sync(0xffffffffu, before, d);
        total += __shfl_xor_sync(0xffffffffu, total, d);
    }
    if (lane == 0) { sm_before[warp] = before; sm_total[warp] = total; }
    __syncthreads();
    before = (sm_before[0] + sm_before[1]) + (sm_before[2] + sm_before[3]);
    total = (sm_total[0] + sm_total[1]) + (sm_total[2] + sm_total[3]);
    const int n_tiles = ad_tiles<16 * AD_UNITS>(ad_len(a, i, nullptr));
    const bool mine = hq < a.n_head;
    RT *out = (RT *)a.out.data + i * a.out.row_stride + (mine ? hq : 0) * a.out.head_stride;
    int w0 = 0, w1 = 0, hg = 0;
    if (n_tiles > 0) {
        const int pairs = a.c.n_kv_head * a.chunks, h = (mine ? hq : 0) / a.group;
        hg = (mine ? hq : 0) - h * a.group;
        const long long T = total * pairs, b0 = before * pairs + (long long)(h * a.chunks + hg / AD_HC) * ad_places(n_tiles), b1 = b0 + n_tiles;
        const int W = ad_warps(a, T);
        w0 = (int)(((b0 + 1) * W - 1) / T); // shares that hold the first and the last tile
        w1 = (int)((b1 * W - 1) / T);
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (n_tiles == 0) {
        if (mine && part_no == 0)
            for (int e = lane; e < HD; e += 32) out[e] = (RT)0.f;
        return;
    }
    if (!mine || w0 == w1) return; // the same for all warps of a head
    float m = -INFINITY, l = 0.f, o[EPL];
#pragma unroll
    for (int e = 0; e < EPL; ++e) o[e] = 0.f;
    const int per = (w1 - w0 + NW) / NW, my0 = w0 + part_no * per, my1 = min(w1, my0 + per - 1); // this warp's shares
    auto part = [&](int w) { return a.part + (((size_t)w * 2 + (w > w0 ? 0 : 1)) * a.hc + hg % AD_HC) * (HD + 4); }; // of share w
    auto fetch = [&](float (&y)[EPL], int w) {
        const float *p = part(min(w, my1));
#pragma unroll
        for (int e = 0; e < EPL; ++e)
            if (HD >= 32 || lane < HD) y[e] = __ldcg(p + lane + 32 * e);
    };
    for (int wb = my0; wb <= my1; wb += 32) { // 32 shares at a time: a lane reads one's statistics ...
        const int w = wb + lane, n = min(32, my1 - wb + 1);
        const bool there = w <= my1;
        const float2 st = there ? __ldcg((const float2 *)(part(w) + HD)) : make_float2(-INFINITY, 0.f);
        float y[AHEAD][EPL];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) fetch(y[j], wb + j);
        float top = st.x;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        const float mn = fmaxf(m, top), ref = mn == -INFINITY ? 0.f : mn;
        const float f_old = ad_exp2(m - ref), g_new = there ? ad_exp2(st.x - ref) : 0.f;
        float sum = there ? st.y * g_new : 0.f;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        l = l * f_old + sum;
        m = mn;
#pragma unroll
        for (int e = 0; e < EPL; ++e) o[e] *= f_old;
        for (int j0 = 0; j0 < n; j0 += AHEAD) { // ... and all of them add up the outputs, AHEAD shares' loads in flight
            float z[AHEAD][EPL];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                const float g = __shfl_sync(0xffffffffu, g_new, (j0 + j) & 31);
#pragma unroll
                for (int e = 0; e < EPL; ++e) z[j][e] = j0 + j < n ? y[j][e] * g : 0.f;
            }
            if (j0 + AHEAD < n) {
#pragma unroll
                for (int j = 0; j < AHEAD; ++j) fetch(y[j], wb + j0 + AHEAD + j);
            }
#pragma unroll
            for (int j = 0; j < AHEAD; ++j)
#pragma unroll
                for (int e = 0; e < EPL; ++e) o[e] += z[j][e];
        }
    }
    if (NW > 1) { // the head's warps, in their order
        if (lane == 0) { sm_m[warp] = m; sm_l[warp] = l; }
#pragma unroll
        for (int e = 0; e < EPL; ++e)
            if (HD >= 32 || lane < HD) sm_o[warp][lane + 32 * e] = o[e];
        __syncthreads();
        if (warp != 0) return;
        for (int w = 1; w < NW; ++w) {
            const float mn = fmaxf(m, sm_m[w]), ref = mn == -INFINITY ? 0.f : mn, f0 = ad_exp2(m - ref), f1 = ad_exp2(sm_m[w] - ref);
            l = l * f0 + sm_l[w] * f1;
            m = mn;
#pragma unroll
            for (int e = 0; e < EPL; ++e)
                if (HD >= 32 || lane < HD) o[e] = o[e] * f0 + sm_o[w][lane + 32 * e] * f1;
        }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int e = 0; e < EPL; ++e)
        if (HD >= 32 || lane < HD) out[lane + 32 * e] = (RT)(o[e] * inv);
}

// ---- host --------------------------------------------------------------------------------------------------------
struct AdPlan { int chunks, hc, n_warps, min_tiles, blocks, whole; int64_t bytes; };

template <int HD> int ad_blocks_hd(int kv_dtype) {
    return kv_dtype == MDI_KV_I8 || kv_dtype == MDI_KV_E4M3 ? AdTile<AD_I8, HD>::BLOCKS : AdTile<AD_F16, HD>::BLOCKS;
}
int ad_blocks(const mdi_kv_cache *c) {
    switch (c->head_dim) {
        case 16: return ad_blocks_hd<16>(c->dtype);
        case 32: return ad_blocks_hd<32>(c->dtype);
        case 64: return ad_blocks_hd<64>(c->dtype);
        default: return ad_blocks_hd<128>(c->dtype);
    }
}

AdPlan ad_plan(const mdi_kv_cache *c, int n_seq, int n_head, int max_len) {
    AdPlan p{};
    const int group = n_head / c->n_kv_head;
    p.chunks = (group + AD_HC - 1) / AD_HC;
    p.hc = std::min(group, AD_HC);
    const int64_t cap = (int64_t)c->pages_per_seq * c->page_tokens, len = max_len > 0 ? std::min<int64_t>(max_len, cap) : cap;
    const int rows = 16 * AD_UNITS;
    const int64_t tiles = (int64_t)std::min(n_seq, AD_MAX_SEQ) * c->n_kv_head * p.chunks * ((len + rows - 1) / rows);
    // a share of fewer tiles would leave more bytes of partial results than it reads
    p.min_tiles = 2 + p.hc / 2;
    const int resident = AD_SM * ad_blocks(c) * AD_WARPS;
    p.n_warps = (int)std::max<int64_t>(1, std::min<int64_t>(resident, tiles / p.min_tiles));
    p.blocks = (p.n_warps + AD_WARPS - 1) / AD_WARPS;
    // Few and short pairs have a cluster of 1 to 8 blocks each to themselves, joined in shared memory: one launch, no workspace, no line
    // of tiles to find a place in.  As many blocks as leave each warp a tile and all pairs room in one wave; not with more than 4 tiles a
    // warp, where equal shares win.  Own blocks / equal shares on the device: 12 heads of 64, f16, 128 rows 3.9 / 7.4 us, 1000 5.8 / 7.8,
    // 4000 9.7 / 10.2; 32 heads of 128, int8, 1000 rows 8.5 / 10.3, 4000 14.1 / 16.3; 8 sequences of 32 heads on 8 of 128, bf16, 128 rows
    // 5.0 / 10.3, 1000 12.6 / 14.0; 192 pairs of 64, 2000 rows 24.2 / 23.9.
    const int64_t n_pairs = (int64_t)n_seq * c->n_kv_head * p.chunks, wave = AD_SM * ad_blocks(c), n_tiles = (len + rows - 1) / rows;
    int own = 8;
    while (own > 1 && (n_pairs * own > wave || AD_WARPS * (own / 2) >= n_tiles)) own /= 2;
    p.whole = n_pairs * own <= wave && n_tiles <= 4 * AD_WARPS * own ? own : 0;
    if (p.whole) return p;
    p.bytes = (int64_t)p.n_warps * 2 * p.hc * (c->head_dim + 4) * 4;
    return p;
}

template <typename RT, int ST, int HD, bool QI> cudaError_t ad_launch_as(const AdArgs &a, int blocks, cudaStream_t st) {
    constexpr size_t smem = AdTile<ST, HD>::BLOCK_SMEM;
    static OpOnce once;
    cudaError_t e = once([] { return cudaFuncSetAttribute(k_attn_decode_op<RT, ST, HD, QI>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem); });
    if (e != cudaSuccess) return e;
    if (a.whole > 1) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(blocks);
        cfg.blockDim = dim3(AD_THREADS);
        cfg.dynamicSmemBytes = smem;
        cfg.stream = st;
        cudaLaunchAttribute at[1];
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim.x = a.whole;
        at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
        cfg.attrs = at;
        cfg.numAttrs = 1;
        return cudaLaunchKernelEx(&cfg, k_attn_decode_op<RT, ST, HD, QI>, a);
    }
    k_attn_decode_op<RT, ST, HD, QI><<<blocks, AD_THREADS, smem, st>>>(a);
    if ((e = cudaGetLastError()) != cudaSuccess || a.whole) return e;
    // many shares per head (few, long sequences): four warps join a head, else one
    const bool wide = a.n_warps > 8 * a.n_seq * a.c.n_kv_head * a.chunks;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(wide ? a.n_head : (a.n_head + 3) / 4, a.n_seq);
    cfg.blockDim = dim3(AD_JOIN_THREADS);
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    return wide ? cudaLaunchKernelEx(&cfg, k_attn_decode_join<RT, HD, 4>, a) : cudaLaunchKernelEx(&cfg, k_attn_decode_join<RT, HD, 1>, a);
}
template <typename RT, int ST, int HD> cudaError_t ad_launch(const AdArgs &a, int blocks, cudaStream_t st) {
    // int8 keys as they are, queries as integers: integers / fp16 planes 361 / 388 us for 64 x 4000 rows of 32 heads of 128 and 80 / 88 us for
    // 12 heads of 64, one head per key head; three heads: 57 / 61 us; four (all that three rows each leave room for): 60 / 58 us
    if constexpr (ST == AD_I8 && HD >= 32)
        if (a.group <= 3) return ad_launch_as<RT, ST, HD, true>(a, blocks, st);
    return ad_launch_as<RT, ST, HD, false>(a, blocks, st);
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
    if (!(scale > 0.f) || scale > 1e38f) return op_fail(MDI_ERR_ARG, "%s: scale must be positive and at most 1e38", who);
    if ((rc = op_check_rows(who, "q", q, n_seq, n_head, false)) != MDI_OK) return rc;
    if ((rc = op_check_rows(who, "out", out, n_seq, n_head, true)) != MDI_OK) return rc;
    if (q->dtype != out->dtype) return op_fail(MDI_ERR_ARG, "%s: q and out differ in dtype", who);
    const AdPlan p = ad_plan(cache, std::max(n_seq, 1), n_head, max_len);
    if (p.bytes > 0 && n_seq > 0 && (!workspace_dev || workspace_bytes < p.bytes || ((uintptr_t)workspace_dev & 15)))
        return op_fail(MDI_ERR_ARG, "%s: needs a 16-byte aligned workspace of %lld bytes", who, (long long)p.bytes);
    if ((rc = op_check_ptrs(who, {{"pool_dev", cache->pool_dev, false}, {"scale_dev", cache->scale_dev, !op_scaled(cache)}, {"page_table_dev", cache->page_table_dev, false},
                                  {"q", q->data_dev, n_seq == 0}, {"out", out->data_dev, n_seq == 0}, {"slot_dev", slot_dev, true},
                                  {"len_dev", len_dev, n_seq == 0}, {"workspace_dev", workspace_dev, true}, {"status_dev", status_dev, true}})) != MDI_OK)
        return rc;
    for (int i0 = 0; i0 < n_seq; i0 += AD_MAX_SEQ) {
        AdArgs a{};
        a.c = op_cache(cache, slot_dev ? slot_dev + i0 : nullptr);
        a.q = op_rows(q); a.out = op_rows(out);
        const int64_t esize = q->dtype == MDI_DTYPE_F32 ? 4 : 2;
        a.q.data += i0 * a.q.row_stride * esize;
        a.out.data += i0 * a.out.row_stride * esize;
        a.len = len_dev + i0; a.status = status_dev;
        a.part = (float *)workspace_dev;
        a.n_seq = std::min(AD_MAX_SEQ, n_seq - i0); a.seq0 = i0;
        a.n_head = n_head; a.group = n_head / cache->n_kv_head;
        a.chunks = p.chunks; a.hc = p.hc; a.n_warps = p.n_warps; a.min_tiles = p.min_tiles; a.whole = p.whole;
        a.scale_log2e = scale * 1.4426950408889634f;
        cudaError_t e;
        OP_ROW_DISPATCH(q->dtype, (e = ad_store<RT>(cache->dtype, a, p.whole ? a.n_seq * cache->n_kv_head * p.chunks * p.whole : p.blocks, (cudaStream_t)stream)));
        if (e != cudaSuccess) return op_cuda(who, e);
    }
    return MDI_OK;
}
