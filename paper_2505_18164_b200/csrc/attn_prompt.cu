// Causal attention over packed sequences (mdi_attn_prompt):
//     out[i][h] = sum_j softmax_j(scale * q[i][h] . K_j) V_j over the keys j <= i + n_k - n_q of i's sequence.
//
// Bound: the tensor cores (4 head_dim flops per query, head and key seen) and, at head_dim 64 and close behind at 128, the
// exponentials (one per query, head and key, 16 a clock and SM).
//
// A block per SM takes items one after the other: two sub-tiles of 128 query rows each, whose keys it walks in tiles of 128, once.  They
// are the same rows of two heads where an even number of heads share a key/value head (both then see the same keys, and short
// sequences fill both: 16 sequences of 1 to 2048 rows, 32 heads on 8, 143 instead of 149 us; 8192 rows 514 instead of 536), else 256
// rows of one head.  Its warps have their own loops over the items, so that loads and products of the next item run while the outputs of
// the last one are still being written (a block per item spends 9000 clocks on filling and emptying itself, three tiles' worth):
//   warp 19     looks items up, ahead of the others;
//   warp 16     requests the tiles by TMA (128-byte swizzle, no multicast): queries once, then keys and values through one ring;
//   warps 17, 18 issue tcgen05.mma, accumulators in tensor memory: one the scores S = Q K^T (128 x 128), the other the outputs O += P V.
//               Both sub-tiles share one S: it is in use only until the softmax has taken the scores into registers, and the next
//               ones are asked for at once, so they are there when a softmax has done its tile; none waits for a product of weights
//               and values.  It also keeps the sub-tiles out of step, so that one's products run while the other's exponentials do (an
//               S each, where head_dim 64 leaves room for it: 462 instead of 419 us for 8192 tokens and 32 heads).
//   warps 0-7, 8-15  softmax of sub-tile 0 and 1.  A row belongs to two threads, 64 keys of a tile each (with one thread per row the
//               schedulers have two warps each and wait for latencies): maximum and sum in fp32, weights rounded to the type of V
//               into tensor memory (an A operand is read from there) in two steps, so that the product of the first half runs while
//               the second is computed.  Weights refer to a maximum that both threads of a row hold; it moves, and what has been
//               summed in O is rescaled, only when a score exceeds it by 2^8 (weights stay below that; sums are fp32), so the two
//               threads hardly ever exchange more than a vote and O hardly ever leaves tensor memory.
//
// Masked places: scores of keys a row does not see are replaced, so whatever they hold has no effect.  Values meet a weight of
// zero, which an infinity or a NaN would survive: in the tiles where anything is masked, such values are replaced by zero in
// shared memory, and the rows that do see them add them at the end (a rare, slow path).
//
// Head dims of 16 and 32 are padded to 64 by TMA (zeros outside the tensor).  Every wait is bounded in wall time; when one runs
// out the block stops waiting, lets its copies land, frees its tensor memory and reports MDI_STATUS_TIMEOUT.
//
// Measured: 8192 tokens, 32 heads on 8 of 128, bf16: 511 us, 1075 TFLOP/s of what is seen, at the 1.6 GHz that the power limit leaves
// (tensor pipe and exponential unit 65% busy each); 16 ragged prompts up to 2048: 143 us, 646 TFLOP/s (some 5 us an item for filling and
// emptying it); 512 rows behind 4096 and three shorter, 32 heads: 79 us, the time of its longest items (64 on 148 SMs).
#include "ops_common.cuh"
#include "tc_prims.cuh"

#include <algorithm>
#include <type_traits>

namespace mdi {
namespace {

constexpr int AP_ROWS = 128;              // rows of a sub-tile, keys of a tile
constexpr int AP_THREADS = 640;
constexpr int AP_SM = 148;                // blocks: one per SM
constexpr int AP_SORT = 64;               // up to this many sequences their tiles are taken in order of the keys they see
constexpr unsigned long long AP_WAIT_NS = 2000000000ull, AP_WAIT_KEY_NS = 100; // longest wait: this, and that per key (some warps wait for the end of an item; a key takes 10 to 20 ns)

struct ApArgs {
    OpRows v, out;
    const int *q_start, *k_start;
    int *status;
    int n_seq, n_q, n_k, group, hd;
    int tile_rows, item_heads, heads; // rows of a sequence and heads of an item; items per tile of rows
    int q_swap, k_swap, v_swap; // the tensor map has (element, row, head) instead of (element, head, row)
    float scale_log2e;
    unsigned long long wait_ns; // longest wait
};

template <int HDP> struct ApLayout {
    static constexpr int TILE = AP_ROWS * HDP * 2;
    static constexpr int STAGES = HDP == 128 ? 4 : 8;
    // columns of tensor memory: scores, weights of sub-tile s at P + 64 s, outputs at O + HDP s
    static constexpr int P = 128, O = 256;
    static constexpr int Q = 0, RING = 2 * TILE, OUT = RING + STAGES * TILE, BARS = OUT + 16 * 2048; // OUT: 2 KB per softmax warp
    static constexpr int SMEM = BARS + 2560; // barriers and what threads tell each other
};

struct ApItem {
    int tile, q0, nq, k0, nk, kvh;         // a tile of a sequence (negative: no more items), the sequence, the key/value head
    int head[2], row[2], n[2];             // of the sub-tiles: head, first row within the sequence, tiles of keys
};
struct ApShared { // behind the ring
    unsigned long long qfull, qempty, full[8], empty[8], sready[2], sfree, pready[4], pvdone[2], ofree[2], ifull[2], iempty[2], drain[2];
    unsigned tmem;
    int abort, poison[4];          // poison: items (number + 1, by number mod 4) with values that had to be replaced
    ApItem item[2];
    float row[2][2][AP_ROWS];      // [sub-tile][half][row]: what the two threads of a row tell each other
};
static_assert(sizeof(ApShared) <= 2560, "ApShared");

__device__ __forceinline__ void ap_init(uint32_t bar, int n) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(n) : "memory"); }
__device__ __forceinline__ void ap_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void ap_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// false: the wait gave up, or another one of the block did.  SLEEP: the thread may sleep between its looks; waking up then takes some
// 180 clocks longer, but a sleeping warp takes no issue slots from the softmax warps of the other sub-tile.
template <bool SLEEP> __device__ __noinline__ bool ap_wait_slow(uint32_t bar, uint32_t parity, int *abort, int *status, unsigned long long wait_ns) {
    const unsigned long long t0 = tg_now();
    for (unsigned it = 0;; ++it) {
        if (SLEEP) {
            uint32_t done;
            asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n selp.u32 %0, 1, 0, p;\n}\n"
                         : "=r"(done) : "r"(bar), "r"(parity), "r"(20000) : "memory"); // ns
            if (done) return true;
        } else if (tg_try_wait(bar, parity)) return true;
        if (SLEEP || (it & 15u) == 15u) {
            if (*(volatile int *)abort) return false;
            if (tg_now() - t0 > wait_ns) break;
        }
    }
    *(volatile int *)abort = 1;
    op_status(status, MDI_STATUS_TIMEOUT);
    return false;
}
__device__ __forceinline__ void ap_tma(uint32_t dst, const CUtensorMap *map, int c0, int c1, int c2, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(bar) : "memory");
}
// 128 rows of one head, HDP elements wide, as HDP / 64 boxes
template <int HDP> __device__ __forceinline__ void ap_load(uint32_t dst, const CUtensorMap *map, int swapped, int head, int row, uint32_t bar) {
#pragma unroll
    for (int b = 0; b < HDP / 64; ++b) ap_tma(dst + b * (AP_ROWS * 128), map, b * 64, swapped ? row : head, swapped ? head : row, bar);
}
// ---- issued by a whole warp in step (one elected lane): the compiler can then keep descriptors in uniform registers; with one
// thread of a diverged warp issuing, moving them there took longer than the products (90 instead of 64 clocks each)
template <bool SLEEP = true> __device__ __forceinline__ bool ap_wait_warp(uint32_t bar, uint32_t parity, int *abort, const ApArgs &a) {
    bool ok = tg_try_wait(bar, parity);
    if (!__all_sync(0xffffffffu, ok)) ok = ok || ap_wait_slow<SLEEP>(bar, parity, abort, a.status, a.wait_ns);
    return __all_sync(0xffffffffu, ok);
}
// named barriers of the softmax warps
__device__ __forceinline__ void ap_meet(int bar, int threads) { asm volatile("barrier.cta.sync %0, %1;" ::"r"(bar), "r"(threads) : "memory"); }
__device__ __forceinline__ bool ap_vote(int bar, bool yes, int threads) { // does any of them say yes?
    int any;
    asm volatile("{\n .reg .pred p, q;\n setp.ne.b32 q, %1, 0;\n barrier.cta.red.or.pred p, %2, %3, q;\n selp.b32 %0, 1, 0, p;\n}\n"
                 : "=r"(any) : "r"((int)yes), "r"(bar), "r"(threads) : "memory");
    return any != 0;
}
// Shared-memory descriptors.  Queries and keys: rows of 128 bytes along head_dim, 128-byte swizzle, 8 rows = 1024 bytes.  Values: the
// rows run along the reduction (keys), the next 64 elements of head_dim are one box further.
__device__ __forceinline__ uint64_t ap_desc(uint32_t addr) {
    return ((uint64_t)(1u << 14 | 1024 >> 4 | 2u << 29) << 32) | 1u << 16 | addr >> 4; // version 1, swizzle 2; addr < 2^18
}
__device__ __forceinline__ uint64_t ap_desc_mn(uint32_t addr) {
    return ((uint64_t)(1u << 14 | 1024 >> 4 | 2u << 29) << 32) | (uint32_t)((AP_ROWS * 128) >> 4) << 16 | addr >> 4;
}
__device__ __forceinline__ void ap_mma_ss(uint32_t d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n .reg .pred p, e;\n elect.sync _|e, 0xffffffff;\n setp.ne.b32 p, %4, 0;\n @e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n"
                 ::"r"(d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void ap_mma_ts(uint32_t d, uint32_t a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n .reg .pred p, e;\n elect.sync _|e, 0xffffffff;\n setp.ne.b32 p, %4, 0;\n @e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n"
                 ::"r"(d), "r"(a), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void ap_commit(uint32_t bar) {
    asm volatile("{\n .reg .pred e;\n elect.sync _|e, 0xffffffff;\n @e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}\n" ::"r"(bar) : "memory");
}
#define AP_R32(r, o) "=r"(r[o]), "=r"(r[o + 1]), "=r"(r[o + 2]), "=r"(r[o + 3]), "=r"(r[o + 4]), "=r"(r[o + 5]), "=r"(r[o + 6]), "=r"(r[o + 7]), \
    "=r"(r[o + 8]), "=r"(r[o + 9]), "=r"(r[o + 10]), "=r"(r[o + 11]), "=r"(r[o + 12]), "=r"(r[o + 13]), "=r"(r[o + 14]), "=r"(r[o + 15]), \
    "=r"(r[o + 16]), "=r"(r[o + 17]), "=r"(r[o + 18]), "=r"(r[o + 19]), "=r"(r[o + 20]), "=r"(r[o + 21]), "=r"(r[o + 22]), "=r"(r[o + 23]), \
    "=r"(r[o + 24]), "=r"(r[o + 25]), "=r"(r[o + 26]), "=r"(r[o + 27]), "=r"(r[o + 28]), "=r"(r[o + 29]), "=r"(r[o + 30]), "=r"(r[o + 31])
#define AP_W32(r, o) "r"(r[o]), "r"(r[o + 1]), "r"(r[o + 2]), "r"(r[o + 3]), "r"(r[o + 4]), "r"(r[o + 5]), "r"(r[o + 6]), "r"(r[o + 7]), \
    "r"(r[o + 8]), "r"(r[o + 9]), "r"(r[o + 10]), "r"(r[o + 11]), "r"(r[o + 12]), "r"(r[o + 13]), "r"(r[o + 14]), "r"(r[o + 15]), \
    "r"(r[o + 16]), "r"(r[o + 17]), "r"(r[o + 18]), "r"(r[o + 19]), "r"(r[o + 20]), "r"(r[o + 21]), "r"(r[o + 22]), "r"(r[o + 23]), \
    "r"(r[o + 24]), "r"(r[o + 25]), "r"(r[o + 26]), "r"(r[o + 27]), "r"(r[o + 28]), "r"(r[o + 29]), "r"(r[o + 30]), "r"(r[o + 31])
// 32 columns of this warp's 32 lanes
template <int N> __device__ __forceinline__ void ap_ld32(uint32_t (&r)[N], int o, uint32_t addr) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,"
                 "%24,%25,%26,%27,%28,%29,%30,%31}, [%32];" : AP_R32(r, o) : "r"(addr) : "memory");
}
template <int N> __device__ __forceinline__ void ap_st32(uint32_t addr, const uint32_t (&r)[N], int o) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,"
                 "%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(addr), AP_W32(r, o) : "memory");
}
__device__ __forceinline__ void ap_ld16(uint32_t (&r)[16], uint32_t addr) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                   "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(addr) : "memory");
}
template <int N> __device__ __forceinline__ void ap_st16(uint32_t addr, const uint32_t (&r)[N], int o) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                 ::"r"(addr), "r"(r[o]), "r"(r[o + 1]), "r"(r[o + 2]), "r"(r[o + 3]), "r"(r[o + 4]), "r"(r[o + 5]), "r"(r[o + 6]), "r"(r[o + 7]),
                 "r"(r[o + 8]), "r"(r[o + 9]), "r"(r[o + 10]), "r"(r[o + 11]), "r"(r[o + 12]), "r"(r[o + 13]), "r"(r[o + 14]), "r"(r[o + 15]) : "memory");
}
__device__ __forceinline__ void ap_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void ap_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ float ap_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// pairs of fp32 in one instruction
typedef unsigned long long ap_f2;
__device__ __forceinline__ ap_f2 ap_pair(float a, float b) { ap_f2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ void ap_unpair(ap_f2 p, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p)); }
__device__ __forceinline__ ap_f2 ap_fma2(ap_f2 a, ap_f2 b, ap_f2 c) { ap_f2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ ap_f2 ap_add2(ap_f2 a, ap_f2 b) { ap_f2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ float ap_max_nan(float a, float b, float c) { float r; asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c)); return r; } // NaN if one is

template <typename T> __device__ __forceinline__ uint32_t ap_pack(float x, float y);
template <> __device__ __forceinline__ uint32_t ap_pack<__half>(float x, float y) { const __half2 h = __floats2half2_rn(x, y); return *(const uint32_t *)&h; }
template <> __device__ __forceinline__ uint32_t ap_pack<__nv_bfloat16>(float x, float y) { const __nv_bfloat162 h = __floats2bfloat162_rn(x, y); return *(const uint32_t *)&h; }
// non-zero in bit 15 / 31 where the lower / upper element is an infinity or a NaN
template <typename T> __device__ __forceinline__ uint32_t ap_nonfinite(uint32_t w) {
    return std::is_same<T, __half>::value ? ((w & 0x7c007c00u) + 0x04000400u) & 0x80008000u : ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
}

// Sequence and tile of rows of an item, x-th in the order in which tiles are taken.  One warp.  A sequence whose offsets do not
// fit has no tiles.  Tiles that see the most keys come first, so that no long one is left to run alone at the end: over all
// sequences where there are at most AP_SORT (found by bisection on the number of key tiles), else sequence by sequence.
struct ApSeq { int q0, nq, k0, nk, tiles; };
__device__ __forceinline__ ApSeq ap_seq(const ApArgs &a, int i, bool tell) {
    ApSeq s{};
    if (i >= a.n_seq) return s;
    const int q0 = a.q_start[i], q1 = a.q_start[i + 1], k0 = a.k_start[i], k1 = a.k_start[i + 1];
    if (q0 < 0 || q1 < q0 || q1 > a.n_q || k0 < 0 || k1 < k0 || k1 > a.n_k) {
        if (tell) op_status(a.status, MDI_STATUS_RANGE);
        return s;
    }
    s.q0 = q0; s.nq = q1 - q0; s.k0 = k0; s.nk = k1 - k0;
    s.tiles = (s.nq + a.tile_rows - 1) / a.tile_rows;
    return s;
}
// tiles of the sequence that see at least `level` key tiles (the last ones; tile t sees the keys up to off + tile_rows (t + 1))
__device__ __forceinline__ int ap_at_least(const ApArgs &a, const ApSeq &s, int level) {
    const int keys = (level - 1) * AP_ROWS; // more than this many
    if (level <= 0) return s.tiles;
    if (s.nk <= keys || s.tiles == 0) return 0;
    const int first = keys - (s.nk - s.nq) < 0 ? 0 : (keys - (s.nk - s.nq)) / a.tile_rows;
    return s.tiles - min(first, s.tiles - 1);
}
__device__ __forceinline__ int ap_sum(int n) { return __reduce_add_sync(0xffffffffu, n); }
__device__ __forceinline__ int ap_scan(int n, int lane) { // sum over the lanes up to this one
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, n, o);
        if (lane >= o) n += up;
    }
    return n;
}
__device__ __forceinline__ void ap_found(ApItem *it, const ApSeq &s, int tile) {
    it->tile = tile; it->q0 = s.q0; it->nq = s.nq; it->k0 = s.k0; it->nk = s.nk;
}
__device__ __forceinline__ void ap_find_tile(const ApArgs &a, int x, int lane, bool tell, ApItem *it) {
    if (lane == 0) it->tile = -1;
    __syncwarp();
    if (a.n_seq <= AP_SORT) {
        const ApSeq s0 = ap_seq(a, lane, tell), s1 = ap_seq(a, lane + 32, tell);
        if (x >= ap_sum(s0.tiles + s1.tiles)) return;
        int lo = 0, hi = (__reduce_max_sync(0xffffffffu, max(s0.nk, s1.nk)) + AP_ROWS - 1) / AP_ROWS; // the largest level with more than x tiles at or above it
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (ap_sum(ap_at_least(a, s0, mid) + ap_at_least(a, s1, mid)) > x) lo = mid; else hi = mid - 1;
        }
        const int a0 = ap_at_least(a, s0, lo), a1 = ap_at_least(a, s1, lo), n0 = a0 - ap_at_least(a, s0, lo + 1), n1 = a1 - ap_at_least(a, s1, lo + 1);
        const int rank = x - (ap_sum(a0 + a1) - ap_sum(n0 + n1)); // among the tiles of exactly this level
        const int before = ap_scan(n0 + n1, lane) - n0 - n1;
        if (rank >= before && rank < before + n0) ap_found(it, s0, s0.tiles - a0 + rank - before);
        else if (rank >= before + n0 && rank < before + n0 + n1) ap_found(it, s1, s1.tiles - a1 + rank - before - n0);
    } else {
        long long total = 0;
        for (int b = 0; b < a.n_seq; b += 32) total += ap_sum(ap_seq(a, b + lane, tell).tiles);
        const long long at = total - 1 - x;
        long long before = 0;
        for (int b = 0; b < a.n_seq && before <= at; b += 32) {
            const ApSeq s = ap_seq(a, b + lane, false);
            const int incl = ap_scan(s.tiles, lane);
            const long long lo = before + incl - s.tiles;
            if (lo <= at && at < lo + s.tiles) ap_found(it, s, (int)(at - lo));
            before += __shfl_sync(0xffffffffu, incl, 31);
        }
    }
}

// The infinities and NaN among the values of key rows j0 .. j1 - 1 in columns o .. o + 31, added to a row's staged outputs.
template <typename T> __device__ __noinline__ void ap_add_nonfinite(const ApArgs &a, unsigned char *line, int swizzle, int kvh, int j0, int j1, int o) {
    const unsigned short *v = (const unsigned short *)a.v.data + kvh * a.v.head_stride + o;
    for (int j = j0; j < j1; ++j)
        for (int e = 0; e < 32 && o + e < a.hd; ++e) {
            const unsigned short w = v[j * a.v.row_stride + e];
            if (!(ap_nonfinite<T>(w) & 0x8000u)) continue;
            T x, *y = (T *)(line + ((e / 8 ^ swizzle) * 16)) + e % 8;
            *(unsigned short *)&x = w;
            *y = (T)((float)*y + (float)x);
        }
}

template <typename T, int HDP>
__global__ void __launch_bounds__(AP_THREADS, 1)
k_attn_prompt(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ ApArgs a) {
    using L = ApLayout<HDP>;
    constexpr bool BF = std::is_same<T, __nv_bfloat16>::value;
    constexpr int NST = L::STAGES;
    extern __shared__ __align__(1024) unsigned char smem[]; // swizzled tiles: 1024-byte aligned (there is no static shared memory)
    ApShared *sh = reinterpret_cast<ApShared *>(smem + L::BARS);
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    const uint32_t s_base = tg_smem_u32(smem);
    const uint32_t b_qfull = tg_smem_u32(&sh->qfull), b_full = tg_smem_u32(sh->full), b_empty = tg_smem_u32(sh->empty), b_s = tg_smem_u32(sh->sready),
                   b_p = tg_smem_u32(sh->pready), b_pv = tg_smem_u32(sh->pvdone), b_free = tg_smem_u32(&sh->sfree),
                   b_qempty = tg_smem_u32(&sh->qempty), b_ofree = tg_smem_u32(sh->ofree), b_ifull = tg_smem_u32(sh->ifull), b_iempty = tg_smem_u32(sh->iempty);
    if (warp == 17) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tg_smem_u32(&sh->tmem)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (tid == 32) {
        ap_init(b_qfull, 1);
        for (int i = 0; i < NST; ++i) { ap_init(b_full + 8 * i, 1); ap_init(b_empty + 8 * i, 1); }
        for (int i = 0; i < 2; ++i) { ap_init(b_s + 8 * i, 1); ap_init(b_pv + 8 * i, 1); }
        ap_init(b_free, 8);
        ap_init(b_qempty, 1);
        for (int i = 0; i < 2; ++i) { ap_init(b_ofree + 8 * i, 8); ap_init(b_ifull + 8 * i, 1); ap_init(b_iempty + 8 * i, 19); } // 16 softmax warps, TMA, two MMA
        for (int i = 0; i < 2; ++i) ap_init(tg_smem_u32(&sh->drain[i]), 1);
        for (int i = 0; i < 4; ++i) ap_init(b_p + 8 * i, 8); // sub-tile 0 first and second step, sub-tile 1
        sh->abort = 0;
        for (int i = 0; i < 4; ++i) sh->poison[i] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = sh->tmem;
    int *abort = &sh->abort;
    // Every warp waits for an item, reads what it wants of it from shared memory and says when it has (the softmax warps at the item's
    // end: what is held in registers meanwhile would be spilled, and with all this shared memory there is next to no first-level cache
    // behind the spills).
    auto arrived = [&](int it) { return ap_wait_warp(b_ifull + 8 * (it & 1), (it >> 1) & 1, abort, a); };
    auto done_with = [&](int it) {
        __syncwarp();
        if (lane == 0) ap_arrive(b_iempty + 8 * (it & 1));
    };

    if (warp == 19) { // ---- items: the blocks take them in turn, to and fro, so that each gets long and short ones alike
        for (int it = 0;; ++it) {
            if (it >= 2 && !ap_wait_warp(b_iempty + 8 * (it & 1), ((it >> 1) & 1) ^ 1, abort, a)) break;
            const long long x = (long long)it * gridDim.x + (it & 1 ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
            ApItem *i = &sh->item[it & 1];
            ap_find_tile(a, (int)min(x / a.heads, (long long)0x7fffffff), lane, it == 0 && blockIdx.x == 0, i);
            __syncwarp();
            const bool last = i->tile < 0;
            if (lane == 0) {
                const int head = (int)(x % a.heads) * a.item_heads;
                i->kvh = head / a.group;
                for (int s = 0; s < 2; ++s) {
                    const int row = i->tile * a.tile_rows + (a.tile_rows > AP_ROWS ? s * AP_ROWS : 0); // keys: up to what the last row sees
                    const int seen = !last && row < i->nq ? min(i->nk, i->nk - i->nq + min(row + AP_ROWS, i->nq)) : 0, n = seen > 0 ? (seen + AP_ROWS - 1) / AP_ROWS : 0;
                    i->head[s] = head + (a.item_heads > 1 ? s : 0);
                    i->row[s] = row;
                    i->n[s] = n;
                }
                ap_arrive(b_ifull + 8 * (it & 1));
            }
            if (__any_sync(0xffffffffu, last)) break;
        }
    } else if (warp == 16) { // ---- TMA (lane 0; the others only keep step)
        int n = 0, items = 0; // tiles of keys and values requested so far, items with queries
        for (int it = 0;; ++it) {
            if (!arrived(it)) break;
            const ApItem *i_ = &sh->item[it & 1];
            const int nt0 = i_->n[0], nt1 = i_->n[1], n_tiles = max(nt0, nt1), kvh = i_->kvh, head0 = i_->head[0], head1 = i_->head[1], k0 = i_->k0,
                      q_row0 = i_->q0 + i_->row[0], q_row1 = i_->q0 + i_->row[1];
            const bool more = i_->tile >= 0;
            done_with(it);
            if (!more) break;
            bool ok = true;
            for (int i = 0; i < 2 * n_tiles && ok; ++i, ++n) {
                const int st = n % NST;
                if (n >= NST) ok = ap_wait_warp(b_empty + 8 * st, ((n / NST) & 1) ^ 1, abort, a);
                if (!ok) break;
                if (lane == 0) {
                    ap_expect(b_full + 8 * st, L::TILE);
                    const uint32_t dst = s_base + L::RING + st * L::TILE;
                    const int row = k0 + (i >> 1) * AP_ROWS;
                    if (i & 1) ap_load<HDP>(dst, &tm_v, a.v_swap, kvh, row, b_full + 8 * st);
                    else ap_load<HDP>(dst, &tm_k, a.k_swap, kvh, row, b_full + 8 * st);
                }
                if (i == 0) { // the queries, once the previous item's are no longer needed
                    if (items > 0) ok = ap_wait_warp(b_qempty, (items - 1) & 1, abort, a);
                    if (ok && lane == 0) {
                        ap_expect(b_qfull, ((nt0 > 0) + (nt1 > 0)) * L::TILE);
                        if (nt0 > 0) ap_load<HDP>(s_base + L::Q, &tm_q, a.q_swap, head0, q_row0, b_qfull);
                        if (nt1 > 0) ap_load<HDP>(s_base + L::Q + L::TILE, &tm_q, a.q_swap, head1, q_row1, b_qfull);
                    }
                    if (ok) ++items;
                }
            }
            if (!ok) break;
        }
        if (*(volatile int *)abort) { // nothing may land in this memory after the block has gone
            int mine = 0;
            if (items > 0) ap_wait_warp(b_qfull, (items - 1) & 1, &mine, a);
            for (int i = max(0, n - NST); i < n; ++i) ap_wait_warp(b_full + 8 * (i % NST), (i / NST) & 1, &mine, a);
        }
    } else if (warp > 16) { // ---- MMA: the whole warp, see ap_mma_ss
        const uint32_t fmt = (1u << 4) | (BF ? (1u << 7) | (1u << 10) : 0u) | ((uint32_t)(AP_ROWS >> 4) << 24);
        const uint32_t base = __shfl_sync(0xffffffffu, s_base, 0), td = __shfl_sync(0xffffffffu, tmem, 0);
        bool ok = true;
        if (warp == 17) { // scores
            const uint32_t id_s = fmt | ((uint32_t)(AP_ROWS >> 3) << 17);
            int st = 0, par = 0, uses = 0, items = 0; // ring stage of the tile's keys and its parity; uses of S so far; items with queries
            for (int it = 0; ok; ++it) {
                ok = arrived(it);
                if (!ok) break;
                const int nt0 = __shfl_sync(0xffffffffu, sh->item[it & 1].n[0], 0), nt1 = __shfl_sync(0xffffffffu, sh->item[it & 1].n[1], 0), n_all = max(nt0, nt1);
                const bool last = __any_sync(0xffffffffu, sh->item[it & 1].tile < 0);
                done_with(it);
                if (last) break;
                if (n_all == 0) continue;
                ok = ap_wait_warp(b_qfull, items++ & 1, abort, a);
                for (int j = 0; j < n_all && ok; ++j) {
                    ok = ap_wait_warp(b_full + 8 * st, par, abort, a);
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        if (j >= (s ? nt1 : nt0) || !ok) continue;
                        if (uses > 0) ok = ap_wait_warp<false>(b_free, (uses - 1) & 1, abort, a); // the previous scores have been taken
                        if (!ok) continue;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        const uint32_t q = base + L::Q + s * L::TILE, k = base + L::RING + st * L::TILE;
#pragma unroll
                        for (int e = 0; e < HDP / 16; ++e) {
                            const uint32_t o = (e / 4) * (AP_ROWS * 128) + (e % 4) * 32;
                            ap_mma_ss(td, ap_desc(q + o), ap_desc(k + o), id_s, e > 0);
                        }
                        ap_commit(b_s + 8 * s);
                        ++uses;
                    }
                    if (!ok) break;
                    ap_commit(b_empty + 8 * st);
                    st += 2;
                    if (st >= NST) { st -= NST; par ^= 1; }
                }
                if (ok) ap_commit(b_qempty);
            }
        } else { // outputs
            const uint32_t id_o = fmt | (1u << 16) | ((uint32_t)(HDP >> 3) << 17);
            int st = 1, par = 0, tiles[2] = {0, 0}, items[2] = {0, 0}; // of each sub-tile so far
            for (int it = 0; ok; ++it) {
                ok = arrived(it);
                if (!ok) break;
                const int nt0 = __shfl_sync(0xffffffffu, sh->item[it & 1].n[0], 0), nt1 = __shfl_sync(0xffffffffu, sh->item[it & 1].n[1], 0), n_all = max(nt0, nt1);
                const bool last = __any_sync(0xffffffffu, sh->item[it & 1].tile < 0);
                done_with(it);
                if (last) break;
                for (int j = 0; j < n_all && ok; ++j) {
                    ok = ap_wait_warp(b_full + 8 * st, par, abort, a);
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        if (j >= (s ? nt1 : nt0)) continue;
                        const uint32_t v = base + L::RING + st * L::TILE;
                        if (j == 0) { // the outputs of the sub-tile's previous item have been taken
                            if (items[s] > 0) ok = ok && ap_wait_warp<false>(b_ofree + 8 * s, (items[s] - 1) & 1, abort, a);
                            ++items[s];
                        }
                        // weights of the keys 0-31 and 64-95, then of the others
#pragma unroll
                        for (int step = 0; step < 2; ++step) {
                            ok = ok && ap_wait_warp<false>(b_p + 16 * s + 8 * step, tiles[s] & 1, abort, a);
                            if (!ok) break;
                            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const int e = 2 * step + (i & 1) + (i >> 1) * 4; // 16 keys
                                ap_mma_ts(td + L::O + s * HDP, td + L::P + s * 64 + e * 8, ap_desc_mn(v + e * 2048), id_o, j > 0 || step > 0 || i > 0);
                            }
                        }
                        ++tiles[s];
                        if (ok) ap_commit(b_pv + 8 * s);
                    }
                    if (!ok) break;
                    ap_commit(b_empty + 8 * st);
                    st += 2;
                    if (st >= NST) { st -= NST; par ^= 1; }
                }
            }
        }
        if (!ok) { // no product may still run when the block goes
            int mine = 0;
            ap_commit(tg_smem_u32(&sh->drain[warp - 17]));
            ap_wait_warp(tg_smem_u32(&sh->drain[warp - 17]), 0, &mine, a);
        }
    } else {
        // ---- softmax: sub-tile s, half of the keys of a tile; thread = row = tensor memory lane
        const int s = warp >> 3, half = (warp >> 2) & 1, r = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)(warp & 3) << 21, t_s = tmem + lanes + 64 * half, t_p = tmem + lanes + L::P + s * 64 + 32 * half, t_o = tmem + lanes + L::O + s * HDP;
        const int two = 1 + s * 4 + (warp & 3);  // named barrier of the two warps that share 32 rows
        // Few registers are left beside a row's 64 scores: what can be read again from shared memory is.
        int t = 0, ring = 1;                     // tiles of this sub-tile so far; place in the ring (counted on) of the values of the tile `t`
        for (int it = 0;; ++it) {
            bool ok = arrived(it);
            const ApItem *item = &sh->item[it & 1];
            if (ap_vote(9 + s, !ok, 256) || item->tile < 0) break; // all of the sub-tile's warps go on, or none
            const int t_end = t + item->n[s];
            int here = min(item->nk - item->nq + item->row[s] + r + 1, item->nk) - 64 * half; // keys of this half and on that the row sees
            // first tile with a key that some row of the item does not see
            const int t_masked = t + min(max(item->nk - item->nq + item->row[0] + 1, 0), item->nk) / AP_ROWS;
            bool first = true;
            float m = -INFINITY, l = 0.f; // what the weights refer to (in log2 units), sum of this thread's weights
            for (; t < t_end; ++t, here -= AP_ROWS, ring += 2) {
                // (after a wait that ran out a warp goes on to meet its partner at the barriers, and does nothing else)
                ok = ok && ap_wait_warp(b_s + 8 * s, t & 1, abort, a);
                if (!ok) {
                    if (ap_vote(two, false, 64)) { ap_meet(two, 64); ap_meet(two, 64); }
                    first = false;
                    continue;
                }
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                uint32_t x[64];
                ap_ld32(x, 0, t_s);
                ap_ld32(x, 32, t_s + 32);
                ap_wait_ld();
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) ap_arrive(b_free); // S may hold the other sub-tile's scores
                if (__any_sync(0xffffffffu, here < 64)) {
#pragma unroll
                    for (int e = 0; e < 64; ++e)
                        if (e >= here) x[e] = 0xff800000u;
                }
                float t4[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) t4[u] = ap_max_nan(__uint_as_float(x[u]), __uint_as_float(x[4 + u]), __uint_as_float(x[8 + u]));
#pragma unroll
                for (int e = 12; e < 60; e += 8)
#pragma unroll
                    for (int u = 0; u < 4; ++u) t4[u] = ap_max_nan(t4[u], __uint_as_float(x[e + u]), __uint_as_float(x[e + 4 + u]));
#pragma unroll
                for (int u = 0; u < 4; ++u) t4[u] = ap_max_nan(t4[u], __uint_as_float(x[60 + u]), t4[u]);
                float top = ap_max_nan(ap_max_nan(t4[0], t4[1], t4[2]), t4[3], t4[3]);
                if (!(top < INFINITY)) l = __uint_as_float(0x7fc00000u); // a score of +inf or NaN: the row is NaN
                // does any row of the two warps need another reference?
                const float c = a.scale_log2e;
                const bool rise = m == -INFINITY ? top > -INFINITY : top * c - m > 8.f;
                if (ap_vote(two, rise, 64)) {
                    sh->row[s][half][r] = top;
                    ap_meet(two, 64);
                    const float other = sh->row[s][half ^ 1][r], high = fmaxf(top, other); // (a NaN is dropped: its row's sum is NaN already)
                    const bool up = m == -INFINITY ? high > -INFINITY : high * c - m > 8.f;
                    const float f = up ? (m == -INFINITY ? 0.f : ap_exp2(m - high * c)) : 1.f;
                    if (up) m = high * c;
                    l *= f;
                    if (!first) { // half of O's columns each, once the product of the previous tile is in
                        ok = ap_wait_warp(b_pv + 8 * s, (t - 1) & 1, abort, a);
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll 1
                        for (int o = half * (HDP / 2); o < (half + 1) * (HDP / 2); o += 16) { // (16 at a time: the 64 scores are held meanwhile)
                            uint32_t y[16];
                            ap_ld16(y, t_o + o);
                            ap_wait_ld();
#pragma unroll
                            for (int e = 0; e < 16; ++e) y[e] = __float_as_uint(__uint_as_float(y[e]) * f);
                            ap_st16(t_o + o, y, 0);
                        }
                        ap_wait_st();
                        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                    }
                    ap_meet(two, 64); // O is rescaled, and row[] may be written again
                }
                first = false;
                if (t >= t_masked) { // values of this tile that may meet a weight of zero: infinities and NaN out (the 64 rows of this half)
                    ok = ok && ap_wait_warp(b_full + 8 * (ring % NST), (ring / NST) & 1, abort, a);
                    if (!ok) continue;
                    unsigned char *v = smem + L::RING + (ring % NST) * L::TILE + (64 * half + (r >> 1)) * 128; // two threads a row
                    constexpr int PART = HDP / 16; // 16-byte chunks each
                    const int c0 = (r & 1) * PART;
                    uint32_t bad = 0;
#pragma unroll
                    for (int q = 0; q < PART; ++q) {
                        const int ch = c0 + ((q + lane) & (PART - 1));
                        const uint4 w = *(const uint4 *)(v + (ch >> 3) * (AP_ROWS * 128) + (ch & 7) * 16);
                        bad |= ap_nonfinite<T>(w.x) | ap_nonfinite<T>(w.y) | ap_nonfinite<T>(w.z) | ap_nonfinite<T>(w.w);
                    }
                    if (bad) {
                        *(volatile int *)&sh->poison[it & 3] = it + 1;
                        __threadfence_block();
                        for (int q = c0 * 4; q < (c0 + PART) * 4; ++q) {
                            uint32_t *w = (uint32_t *)(v + (q >> 5) * (AP_ROWS * 128)) + (q & 31);
                            const uint32_t f = ap_nonfinite<T>(*w);
                            if (f) *w &= ~((f >> 15) * 0xffffu);
                        }
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    }
                }
                // The previous weights have been used.  (Waiting here rather than before the first store, half an exponential phase later,
                // keeps the sub-tiles out of step: 2990 instead of 3400 clocks a tile.)
                ok = ok && (t == 0 || ap_wait_warp(b_pv + 8 * s, (t - 1) & 1, abort, a));
                if (!ok) continue;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const float ref = m == -INFINITY ? 0.f : m;
                const ap_f2 c2 = ap_pair(c, c), r2 = ap_pair(-ref, -ref);
                ap_f2 sum0 = ap_pair(0.f, 0.f), sum1 = sum0;
                // (Replacing a quarter of the exponentials by polynomials on the multiply-add pipe made a tile 20% slower: the exponential
                // unit is 70% busy, and the softmax warps' instructions, not it, are what the four warps of a scheduler queue for.)
#pragma unroll
                for (int step = 0; step < 2; ++step) {
#pragma unroll
                    for (int e = 32 * step; e < 32 * step + 32; e += 2) {
                        const ap_f2 y = ap_fma2(ap_pair(__uint_as_float(x[e]), __uint_as_float(x[e + 1])), c2, r2);
                        float p0, p1;
                        ap_unpair(y, p0, p1);
                        p0 = ap_exp2(p0);
                        p1 = ap_exp2(p1);
                        if (e % 4) sum1 = ap_add2(sum1, ap_pair(p0, p1)); else sum0 = ap_add2(sum0, ap_pair(p0, p1));
                        x[e / 2] = ap_pack<T>(p0, p1);
                    }
                    ap_st16(t_p + 16 * step, x, 16 * step);
                    ap_wait_st();
                    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) ap_arrive(b_p + 16 * s + 8 * step);
                }
                {
                    float s0, s1;
                    ap_unpair(ap_add2(sum0, sum1), s0, s1);
                    l += s0 + s1;
                }
            }
            const int n_mine = item->n[s];
            ring += 2 * (max(item->n[0], item->n[1]) - n_mine); // the other sub-tile's
            // ---- output: half of the columns each
            const int row = item->row[s] + r, nq = item->nq, seen = min(item->nk - nq + row + 1, item->nk); // row of the sequence
            const bool valid = row < nq;
            T *out = (T *)a.out.data + (long long)(item->q0 + row) * a.out.row_stride + (long long)item->head[s] * a.out.head_stride;
            if (n_mine == 0) {
                if (valid && half == 0)
                    for (int e = 0; e < a.hd; e += 8) *(uint4 *)(out + e) = make_uint4(0, 0, 0, 0);
            } else {
                sh->row[s][half][r] = l;
                ap_meet(9 + s, 256); // the sums; and all of this sub-tile's looks at the values are done
                ok = ok && ap_wait_warp(b_pv + 8 * s, (t - 1) & 1, abort, a);
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                // 32 columns at a time through shared memory, so that stores cover whole sectors side by side: a row per thread, 16 bytes at a
                // time, took 2000 clocks more
                unsigned char *mine = smem + L::OUT + warp * 2048;
                const bool poison = *(volatile int *)&sh->poison[it & 3] == it + 1;
                const float sum = sh->row[s][0][r] + sh->row[s][1][r], inv = seen > 0 && sum != 0.f ? 1.f / sum : 0.f; // (0: all scores are -inf)
#pragma unroll 1
                for (int o = half * (HDP / 2); o < (half + 1) * (HDP / 2) && ok; o += 32) {
                    uint32_t y[32];
                    ap_ld32(y, 0, t_o + o);
                    ap_wait_ld();
#pragma unroll
                    for (int e = 0; e < 32; ++e) y[e] = seen > 0 ? __float_as_uint(__uint_as_float(y[e]) * inv) : 0u;
#pragma unroll
                    for (int e = 0; e < 32; e += 8) {
                        uint4 w;
                        w.x = ap_pack<T>(__uint_as_float(y[e]), __uint_as_float(y[e + 1]));
                        w.y = ap_pack<T>(__uint_as_float(y[e + 2]), __uint_as_float(y[e + 3]));
                        w.z = ap_pack<T>(__uint_as_float(y[e + 4]), __uint_as_float(y[e + 5]));
                        w.w = ap_pack<T>(__uint_as_float(y[e + 6]), __uint_as_float(y[e + 7]));
                        *(uint4 *)(mine + lane * 64 + ((e / 8 ^ (lane >> 1 & 3)) * 16)) = w;
                    }
                    if (poison && valid) ap_add_nonfinite<T>(a, mine + lane * 64, lane >> 1 & 3, item->kvh, item->k0 + min(max(item->nk - nq + item->row[0] + 1, 0), item->nk) / AP_ROWS * AP_ROWS, item->k0 + seen, o);
                    if (o + 32 == (half + 1) * (HDP / 2)) { // the last of this warp's columns: the next item's outputs may come
                        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                        __syncwarp();
                        if (lane == 0) ap_arrive(b_ofree + 8 * s);
                    }
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 4; ++i) { // 32 rows of 4 chunks, four neighbouring lanes on a row
                        const int rr = i * 8 + lane / 4, ch = lane & 3, col = o + ch * 8, to = row - lane + rr;
                        if (to < nq && col < a.hd)
                            *(uint4 *)(out + (long long)(rr - lane) * a.out.row_stride + col) = *(const uint4 *)(mine + rr * 64 + ((ch ^ (rr >> 1 & 3)) * 16));
                    }
                    __syncwarp();
                }
            }
            done_with(it);
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (warp == 17) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    }
}

// ---- host --------------------------------------------------------------------------------------------------------
// Map over [rows][heads][hd] with a box of 64 elements x 1 head x 128 rows; the dimension with the smaller stride first.
CUresult ap_make_map(CUtensorMap *map, const mdi_rows *r, int rows, int heads, int hd, int *swapped) {
    const tg_encode_fn enc = tg_encoder();
    if (!enc) return CUDA_ERROR_NOT_SUPPORTED;
    const cuuint64_t hs = heads > 1 ? (cuuint64_t)r->head_stride * 2 : 0, rs = rows > 1 ? (cuuint64_t)r->row_stride * 2 : 0;
    *swapped = heads > 1 && rows > 1 && hs > rs;
    cuuint64_t dims[3] = {(cuuint64_t)hd, (cuuint64_t)heads, (cuuint64_t)rows}, strides[2] = {hs ? hs : (cuuint64_t)hd * 2, rs ? rs : std::max(hs, (cuuint64_t)hd * 2) * heads};
    cuuint32_t box[3] = {64, 1, (cuuint32_t)AP_ROWS}, estr[3] = {1, 1, 1};
    if (*swapped) {
        std::swap(dims[1], dims[2]);
        std::swap(strides[0], strides[1]);
        std::swap(box[1], box[2]);
    }
    return enc(map, r->dtype == MDI_DTYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, r->data_dev, dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
}

template <typename T, int HDP>
cudaError_t ap_launch(const CUtensorMap &mq, const CUtensorMap &mk, const CUtensorMap &mv, const ApArgs &a, dim3 grid, cudaStream_t st) {
    static OpOnce once;
    if (const cudaError_t e = once([] { return cudaFuncSetAttribute(k_attn_prompt<T, HDP>, cudaFuncAttributeMaxDynamicSharedMemorySize, ApLayout<HDP>::SMEM); })) return e;
    k_attn_prompt<T, HDP><<<grid, AP_THREADS, ApLayout<HDP>::SMEM, st>>>(mq, mk, mv, a);
    return cudaGetLastError();
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
    if (!(scale > 0.f) || scale > 1e38f) return op_fail(MDI_ERR_ARG, "%s: scale must be positive and at most 1e38", who);
    if (n_q_rows > 1 << 30 || n_k_rows > 1 << 30) return op_fail(MDI_ERR_SHAPE, "%s: more than 2^30 rows", who);
    if ((rc = op_check_rows(who, "q", q, n_q_rows, n_head, false)) != MDI_OK) return rc;
    if ((rc = op_check_rows(who, "k", k, n_k_rows, n_kv_head, false)) != MDI_OK) return rc;
    if ((rc = op_check_rows(who, "v", v, n_k_rows, n_kv_head, false)) != MDI_OK) return rc;
    if ((rc = op_check_rows(who, "out", out, n_q_rows, n_head, true)) != MDI_OK) return rc;
    if ((q->dtype != MDI_DTYPE_F16 && q->dtype != MDI_DTYPE_BF16) || k->dtype != q->dtype || v->dtype != q->dtype || out->dtype != q->dtype)
        return op_fail(MDI_ERR_ARG, "%s: q, k, v and out must share one dtype, F16 or BF16", who);
    if ((rc = op_check_ptrs(who, {{"q", q->data_dev, n_q_rows == 0}, {"k", k->data_dev, n_k_rows == 0}, {"v", v->data_dev, n_k_rows == 0}, {"out", out->data_dev, n_q_rows == 0},
                                  {"q_start_dev", q_start_dev, n_seq == 0}, {"k_start_dev", k_start_dev, n_seq == 0}, {"status_dev", status_dev, true}})) != MDI_OK)
        return rc;
    for (const mdi_rows *r : {q, k, v})
        if ((r->row_stride == 0 && (r == q ? n_q_rows : n_k_rows) > 1) || (r->head_stride == 0 && (r == q ? n_head : n_kv_head) > 1))
            return op_fail(MDI_ERR_SHAPE, "%s: strides of q, k and v must not be zero", who);
    if (n_seq == 0 || n_q_rows == 0) return MDI_OK;
    ApArgs a{};
    CUtensorMap mq, mk, mv;
    // without keys nothing is loaded: any valid map will do
    const mdi_rows *mkr = n_k_rows ? k : q, *mvr = n_k_rows ? v : q;
    const int kr = n_k_rows ? n_k_rows : n_q_rows, kh = n_k_rows ? n_kv_head : n_head;
    CUresult e = ap_make_map(&mq, q, n_q_rows, n_head, head_dim, &a.q_swap);
    if (e == CUDA_SUCCESS) e = ap_make_map(&mk, mkr, kr, kh, head_dim, &a.k_swap);
    if (e == CUDA_SUCCESS) e = ap_make_map(&mv, mvr, kr, kh, head_dim, &a.v_swap);
    if (e != CUDA_SUCCESS) return op_fail(MDI_ERR_SHAPE, "%s: no tensor map for these rows and strides (%d)", who, (int)e);
    a.v = op_rows(v); a.out = op_rows(out);
    a.q_start = q_start_dev; a.k_start = k_start_dev; a.status = status_dev;
    a.n_seq = n_seq; a.n_q = n_q_rows; a.n_k = n_k_rows; a.group = n_head / n_kv_head; a.hd = head_dim;
    a.scale_log2e = scale * 1.4426950408889634f;
    a.wait_ns = AP_WAIT_NS + AP_WAIT_KEY_NS * (unsigned long long)n_k_rows;
    const bool pair = a.group % 2 == 0;
    a.tile_rows = pair ? AP_ROWS : 2 * AP_ROWS;
    a.item_heads = pair ? 2 : 1;
    a.heads = n_head / a.item_heads;
    const int64_t tiles = (int64_t)n_q_rows / a.tile_rows + std::min(n_seq, n_q_rows); // at most
    const dim3 grid((unsigned)std::min<int64_t>(tiles * a.heads, AP_SM));
    cudaStream_t st = (cudaStream_t)stream;
    cudaError_t ce;
    if (q->dtype == MDI_DTYPE_F16) ce = head_dim == 128 ? ap_launch<__half, 128>(mq, mk, mv, a, grid, st) : ap_launch<__half, 64>(mq, mk, mv, a, grid, st);
    else ce = head_dim == 128 ? ap_launch<__nv_bfloat16, 128>(mq, mk, mv, a, grid, st) : ap_launch<__nv_bfloat16, 64>(mq, mk, mv, a, grid, st);
    return op_cuda(who, ce);
}
