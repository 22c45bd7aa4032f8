// Causal attention over packed sequences (mdi_attn_prompt):
//     out[i][h] = sum_j softmax_j(scale * q[i][h] . K_j) V_j over the keys j <= i + n_k - n_q of i's sequence.
//
// Bound: the tensor cores (4 head_dim flops per query, head and key seen) and, at head_dim 64 and close behind at 128, the
// exponentials (one per query, head and key, 16 a clock and SM).
//
// One block takes 256 query rows of one head (two sub-tiles of 128) and walks the keys its rows see in tiles of 128, once:
//   warp 8      requests the tiles by TMA (128-byte swizzle, no multicast): queries once, then keys and values through one ring;
//   warp 9      issues tcgen05.mma: scores S = Q K^T (128 x 128) and outputs O += P V, accumulators in tensor memory.  The
//               sub-tiles alternate, so that one's products run while the other's softmax does;
//   warps 0-3, 4-7  softmax of sub-tile 0 and 1, one row per thread: scores from tensor memory, running maximum and sum in fp32,
//               weights rounded to the type of V back into the tensor memory of the scores (an A operand is read from there).
//               What has been summed in O is rescaled only when a row's maximum rises by more than 2^8 (weights stay below
//               that; sums are fp32), so that the outputs hardly ever leave tensor memory on the way.
// The scores' accumulator ready implies that the sub-tile's previous output product is complete (both are committed in order),
// which is what makes the rescaling safe.
//
// Masked places: scores of keys a row does not see are replaced, so whatever they hold has no effect.  Values meet a weight of
// zero, which an infinity or a NaN would survive: in the tiles where anything is masked, such values are replaced by zero in
// shared memory, and the rows that do see them add them at the end (a rare, slow path).
//
// Head dims of 16 and 32 are padded to 64 by TMA (zeros outside the tensor).  Every wait is bounded in wall time; when one runs
// out the block stops waiting, lets its copies land, frees its tensor memory and reports MDI_STATUS_TIMEOUT.
#include "ops_common.cuh"
#include "tc_prims.cuh"

#include <algorithm>
#include <type_traits>

namespace mdi {
namespace {

constexpr int AP_ROWS = 128;              // rows of a sub-tile, keys of a tile
constexpr int AP_THREADS = 320;
constexpr unsigned long long AP_WAIT_NS = 2000000000ull;

struct ApArgs {
    OpRows v, out;
    const int *q_start, *k_start;
    int *status;
    int n_seq, n_q, n_k, group, hd;
    int q_swap, k_swap, v_swap; // the tensor map has (element, row, head) instead of (element, head, row)
    float scale_log2e;
};

template <int HDP> struct ApLayout {
    static constexpr int TILE = AP_ROWS * HDP * 2;
    static constexpr int STAGES = HDP == 128 ? 5 : 8;
    static constexpr int Q = 0, RING = 2 * TILE, BARS = RING + STAGES * TILE;
    static constexpr int SMEM = BARS + 256 + 1024; // barriers, alignment slack
};

struct ApShared { // behind the ring
    unsigned long long qfull, full[8], empty[8], sready[2], pready[2], odone[2], drain;
    unsigned tmem;
    int abort, poison;
    int seq, tile, q0, nq, k0, nk; // this block's sequence
};
static_assert(sizeof(ApShared) <= 256, "ApShared");

__device__ __forceinline__ void ap_init(uint32_t bar, int n) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(n) : "memory"); }
__device__ __forceinline__ void ap_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void ap_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// false: the wait gave up, or another one of the block did
__device__ __noinline__ bool ap_wait_slow(uint32_t bar, uint32_t parity, int *abort, int *status) {
    const unsigned long long t0 = tg_now();
    for (unsigned it = 0;; ++it) {
        if (tg_try_wait(bar, parity)) return true;
        if ((it & 15u) == 15u) {
            if (*(volatile int *)abort) return false;
            if (tg_now() - t0 > AP_WAIT_NS) break;
        }
    }
    *(volatile int *)abort = 1;
    op_status(status, MDI_STATUS_TIMEOUT);
    return false;
}
__device__ __forceinline__ bool ap_wait(uint32_t bar, uint32_t parity, int *abort, int *status) {
    return tg_try_wait(bar, parity) || ap_wait_slow(bar, parity, abort, status);
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
// Descriptor of an operand whose rows run along the reduction (values: [key][64 elements of head_dim], 128 bytes a key, swizzled):
// 8 keys = 1024 bytes, the next 64 elements of head_dim one box further.
__device__ __forceinline__ uint64_t ap_desc_mn(uint32_t addr) {
    uint64_t d = 0;
    d |= (uint64_t)((addr & 0x3FFFF) >> 4);
    d |= (uint64_t)((AP_ROWS * 128) >> 4) << 16;
    d |= (uint64_t)(1024 >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}
__device__ __forceinline__ void ap_mma_ts(uint32_t d, uint32_t a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n"
                 ::"r"(d), "r"(a), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
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
__device__ __forceinline__ void ap_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void ap_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ float ap_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

template <typename T> __device__ __forceinline__ uint32_t ap_pack(float x, float y);
template <> __device__ __forceinline__ uint32_t ap_pack<__half>(float x, float y) { const __half2 h = __floats2half2_rn(x, y); return *(const uint32_t *)&h; }
template <> __device__ __forceinline__ uint32_t ap_pack<__nv_bfloat16>(float x, float y) { const __nv_bfloat162 h = __floats2bfloat162_rn(x, y); return *(const uint32_t *)&h; }
// non-zero in bit 15 / 31 where the lower / upper element is an infinity or a NaN
template <typename T> __device__ __forceinline__ uint32_t ap_nonfinite(uint32_t w) {
    return std::is_same<T, __half>::value ? ((w & 0x7c007c00u) + 0x04000400u) & 0x80008000u : ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
}

// Sequence and 256-row tile of the block: the tiles of all sequences end to end, the last one first (it sees the most keys).
// One warp.  A sequence whose offsets do not fit has no tiles.
__device__ __forceinline__ void ap_find_tile(const ApArgs &a, int x, int lane, ApShared *sh) {
    auto tiles_of = [&](int i, bool tell) {
        if (i >= a.n_seq) return 0;
        const int q0 = a.q_start[i], q1 = a.q_start[i + 1], k0 = a.k_start[i], k1 = a.k_start[i + 1];
        const bool bad = q0 < 0 || q1 < q0 || q1 > a.n_q || k0 < 0 || k1 < k0 || k1 > a.n_k;
        if (bad && tell) op_status(a.status, MDI_STATUS_RANGE);
        return bad ? 0 : (q1 - q0 + 2 * AP_ROWS - 1) / (2 * AP_ROWS);
    };
    const bool tell = blockIdx.x == 0 && blockIdx.y == 0;
    long long total = 0;
    for (int b = 0; b < a.n_seq; b += 32) {
        int n = tiles_of(b + lane, tell);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) n += __shfl_xor_sync(0xffffffffu, n, o);
        total += n;
    }
    if (lane == 0) sh->seq = -1;
    __syncwarp();
    const long long at = total - 1 - x;
    if (at < 0) return;
    long long before = 0;
    for (int b = 0; b < a.n_seq && before <= at; b += 32) {
        const int n = tiles_of(b + lane, false);
        int incl = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int up = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += up;
        }
        const long long lo = before + incl - n;
        if (n > 0 && lo <= at && at < lo + n) {
            const int i = b + lane;
            sh->seq = i;
            sh->tile = (int)(at - lo);
            sh->q0 = a.q_start[i];
            sh->nq = a.q_start[i + 1] - a.q_start[i];
            sh->k0 = a.k_start[i];
            sh->nk = a.k_start[i + 1] - a.k_start[i];
        }
        before += __shfl_sync(0xffffffffu, incl, 31);
    }
    __syncwarp();
}

// grid (tiles, n_head)
template <typename T, int HDP>
__global__ void __launch_bounds__(AP_THREADS, 1)
k_attn_prompt(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const ApArgs a) {
    using L = ApLayout<HDP>;
    constexpr bool BF = std::is_same<T, __nv_bfloat16>::value;
    constexpr int NST = L::STAGES;
    extern __shared__ unsigned char ap_raw[];
    unsigned char *smem = reinterpret_cast<unsigned char *>(((uintptr_t)ap_raw + 1023) & ~(uintptr_t)1023);
    ApShared *sh = reinterpret_cast<ApShared *>(smem + L::BARS);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t s_base = tg_smem_u32(smem);
    const uint32_t b_qfull = tg_smem_u32(&sh->qfull), b_full = tg_smem_u32(sh->full), b_empty = tg_smem_u32(sh->empty), b_s = tg_smem_u32(sh->sready),
                   b_p = tg_smem_u32(sh->pready), b_o = tg_smem_u32(sh->odone);
    if (warp == 0) ap_find_tile(a, blockIdx.x, lane, sh);
    if (tid == 32) {
        ap_init(b_qfull, 1);
        ap_init(tg_smem_u32(&sh->drain), 1);
        for (int i = 0; i < NST; ++i) { ap_init(b_full + 8 * i, 1); ap_init(b_empty + 8 * i, 1); }
        for (int i = 0; i < 2; ++i) { ap_init(b_s + 8 * i, 1); ap_init(b_p + 8 * i, 4); ap_init(b_o + 8 * i, 1); }
        sh->abort = 0;
        sh->poison = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    if (sh->seq < 0) return; // no such tile
    const int row0 = sh->tile * 2 * AP_ROWS, nq = sh->nq, nk = sh->nk, q0 = sh->q0, k0 = sh->k0, off = nk - nq;
    const int head = blockIdx.y, kvh = head / a.group;
    // key tiles of each sub-tile: up to what its last row sees
    int nt[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const int r0 = row0 + s * AP_ROWS, seen = r0 < nq ? min(nk, off + min(r0 + AP_ROWS, nq)) : 0;
        nt[s] = seen > 0 ? (seen + AP_ROWS - 1) / AP_ROWS : 0;
    }
    const int n_tiles = max(nt[0], nt[1]);
    const int masked_from = min(max(off + row0 + 1, 0), nk) / AP_ROWS; // first tile with a key that some row of the block does not see
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tg_smem_u32(&sh->tmem)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = sh->tmem; // S0 | S1 | O0 | O1, 128 columns each
    int *abort = &sh->abort;

    if (warp == 8) {
        if (lane == 0 && n_tiles > 0) { // ---- TMA
            ap_expect(b_qfull, ((nt[0] > 0) + (nt[1] > 0)) * L::TILE);
#pragma unroll
            for (int s = 0; s < 2; ++s)
                if (nt[s] > 0) ap_load<HDP>(s_base + L::Q + s * L::TILE, &tm_q, a.q_swap, head, q0 + row0 + s * AP_ROWS, b_qfull);
            int issued = 0;
            for (int n = 0; n < 2 * n_tiles; ++n) {
                const int st = n % NST;
                if (n >= NST && !ap_wait(b_empty + 8 * st, ((n / NST) & 1) ^ 1, abort, a.status)) break;
                ap_expect(b_full + 8 * st, L::TILE);
                const uint32_t dst = s_base + L::RING + st * L::TILE;
                const int row = k0 + (n >> 1) * AP_ROWS;
                if (n & 1) ap_load<HDP>(dst, &tm_v, a.v_swap, kvh, row, b_full + 8 * st);
                else ap_load<HDP>(dst, &tm_k, a.k_swap, kvh, row, b_full + 8 * st);
                issued = n + 1;
            }
            if (*(volatile int *)abort) { // nothing may land in this memory after the block has gone
                int mine = 0;
                ap_wait(b_qfull, 0, &mine, a.status);
                for (int n = max(0, issued - NST); n < issued; ++n) ap_wait(b_full + 8 * (n % NST), (n / NST) & 1, &mine, a.status);
            }
        }
    } else if (warp == 9) {
        if (lane == 0 && n_tiles > 0) { // ---- MMA
            const uint32_t fmt = (1u << 4) | (BF ? (1u << 7) | (1u << 10) : 0u) | ((uint32_t)(AP_ROWS >> 4) << 24);
            const uint32_t id_s = fmt | ((uint32_t)(AP_ROWS >> 3) << 17), id_o = fmt | (1u << 16) | ((uint32_t)(HDP >> 3) << 17);
            auto scores = [&](int s, int j) {
                const uint32_t q = s_base + L::Q + s * L::TILE, k = s_base + L::RING + (2 * j % NST) * L::TILE;
#pragma unroll
                for (int e = 0; e < HDP / 16; ++e) {
                    const uint32_t o = (e / 4) * (AP_ROWS * 128) + (e % 4) * 32;
                    tg_mma(tmem + s * 128, tg_desc(q + o), tg_desc(k + o), id_s, e > 0);
                }
                tg_commit(b_s + 8 * s);
            };
            bool ok = ap_wait(b_qfull, 0, abort, a.status) && ap_wait(b_full, 0, abort, a.status);
            if (ok) {
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                for (int s = 0; s < 2; ++s)
                    if (nt[s] > 0) scores(s, 0);
                tg_commit(b_empty);
            }
            for (int j = 0; j < n_tiles && ok; ++j) {
                const int nv = 2 * j + 1, nk1 = 2 * j + 2;
                ok = ap_wait(b_full + 8 * (nv % NST), (nv / NST) & 1, abort, a.status);
                for (int s = 0; s < 2 && ok; ++s) {
                    if (j >= nt[s]) continue;
                    ok = ap_wait(b_p + 8 * s, j & 1, abort, a.status);
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t v = s_base + L::RING + (nv % NST) * L::TILE;
#pragma unroll
                    for (int e = 0; e < AP_ROWS / 16; ++e)
                        ap_mma_ts(tmem + 256 + s * 128, tmem + s * 128 + e * 8, ap_desc_mn(v + e * 2048), id_o, j > 0 || e > 0);
                    if (j + 1 < nt[s]) {
                        ok = ap_wait(b_full + 8 * (nk1 % NST), (nk1 / NST) & 1, abort, a.status);
                        if (!ok) break;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        scores(s, j + 1);
                    } else tg_commit(b_o + 8 * s);
                }
                if (!ok) break;
                tg_commit(b_empty + 8 * (nv % NST));
                if (j + 1 < n_tiles) tg_commit(b_empty + 8 * (nk1 % NST));
            }
            if (!ok) { // no product may still run when the block goes
                int mine = 0;
                tg_commit(tg_smem_u32(&sh->drain));
                ap_wait(tg_smem_u32(&sh->drain), 0, &mine, a.status);
            }
        }
    } else {
        // ---- softmax: warps 0-3 sub-tile 0, warps 4-7 sub-tile 1; thread = row = tensor memory lane
        const int s = warp >> 2, r = (warp & 3) * 32 + lane, row = row0 + s * AP_ROWS + r; // row of the sequence
        const uint32_t lanes = (uint32_t)(warp & 3) << 21, t_s = tmem + lanes + s * 128, t_o = tmem + lanes + 256 + s * 128;
        const int seen = min(off + row + 1, nk); // keys this row sees (also for rows behind the sequence: never stored)
        const int n_mine = s ? nt[1] : nt[0];
        const float c = a.scale_log2e;
        float m = -INFINITY, l = 0.f; // maximum of the raw scores that the weights refer to, sum of the weights
        bool ok = true;
        for (int j = 0; j < n_mine; ++j) {
            ok = ap_wait(b_s + 8 * s, j & 1, abort, a.status);
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            uint32_t x[128];
            ap_ld32(x, 0, t_s);
            ap_ld32(x, 32, t_s + 32);
            ap_ld32(x, 64, t_s + 64);
            ap_ld32(x, 96, t_s + 96);
            ap_wait_ld();
            const int here = seen - j * AP_ROWS;
            if (__any_sync(0xffffffffu, here < AP_ROWS)) {
#pragma unroll
                for (int e = 0; e < 128; ++e)
                    if (e >= here) x[e] = 0xff800000u;
            }
            float t4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int e = 0; e < 128; e += 8)
#pragma unroll
                for (int u = 0; u < 4; ++u) t4[u] = fmaxf(t4[u], fmaxf(__uint_as_float(x[e + u]), __uint_as_float(x[e + 4 + u])));
            const float top = fmaxf(fmaxf(t4[0], t4[1]), fmaxf(t4[2], t4[3]));
            const bool rise = m == -INFINITY ? top > -INFINITY : (top - m) * c > 8.f;
            if (__any_sync(0xffffffffu, rise)) {
                const float f = rise ? (m == -INFINITY ? 0.f : ap_exp2((m - top) * c)) : 1.f;
                if (rise) m = top;
                l *= f;
                if (j > 0) {
#pragma unroll 1
                    for (int o = 0; o < HDP; o += 32) {
                        uint32_t y[32];
                        ap_ld32(y, 0, t_o + o);
                        ap_wait_ld();
#pragma unroll
                        for (int e = 0; e < 32; ++e) y[e] = __float_as_uint(__uint_as_float(y[e]) * f);
                        ap_st32(t_o + o, y, 0);
                    }
                }
            }
            const float ref = m == -INFINITY ? 0.f : m * c;
            float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int e = 0; e < 128; e += 2) {
                const float p0 = ap_exp2(fmaf(__uint_as_float(x[e]), c, -ref)), p1 = ap_exp2(fmaf(__uint_as_float(x[e + 1]), c, -ref));
                sum[e % 4] += p0;
                sum[e % 4 + 1] += p1;
                x[e / 2] = ap_pack<T>(p0, p1);
            }
            l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
            ap_st32(t_s, x, 0);
            ap_st32(t_s + 32, x, 32);
            if (j >= masked_from) { // values of this tile that may meet a weight of zero: infinities and NaN out
                const int nv = 2 * j + 1;
                ok = ap_wait(b_full + 8 * (nv % NST), (nv / NST) & 1, abort, a.status);
                if (!ok) break;
                unsigned char *v = smem + L::RING + (nv % NST) * L::TILE + r * 128;
#pragma unroll
                for (int b = 0; b < HDP / 64; ++b) {
                    uint32_t bad = 0;
#pragma unroll
                    for (int q = 0; q < 8; ++q) {
                        const uint4 w = *(const uint4 *)(v + b * (AP_ROWS * 128) + ((q ^ lane) & 7) * 16);
                        bad |= ap_nonfinite<T>(w.x) | ap_nonfinite<T>(w.y) | ap_nonfinite<T>(w.z) | ap_nonfinite<T>(w.w);
                    }
                    if (bad) {
                        *(volatile int *)&sh->poison = 1;
                        __threadfence_block();
                        for (int q = 0; q < 32; ++q) {
                            uint32_t *w = (uint32_t *)(v + b * (AP_ROWS * 128)) + q;
                            const uint32_t f = ap_nonfinite<T>(*w);
                            if (f) *w &= ~((f >> 15) * 0xffffu);
                        }
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    }
                }
            }
            ap_wait_st();
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) ap_arrive(b_p + 8 * s);
        }
        // ---- output
        const bool valid = row < nq;
        T *out = (T *)a.out.data + (long long)(q0 + row) * a.out.row_stride + (long long)head * a.out.head_stride;
        if (n_mine == 0) {
            if (valid)
                for (int e = 0; e < a.hd; e += 8) *(uint4 *)(out + e) = make_uint4(0, 0, 0, 0);
        } else if (ok && ap_wait(b_o + 8 * s, 0, abort, a.status)) {
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            asm volatile("bar.sync %0, 128;" ::"r"(1 + s) : "memory"); // all of this sub-tile's looks at the values are done
            const bool poison = *(volatile int *)&sh->poison;
            const float inv = seen > 0 ? 1.f / l : 0.f;
#pragma unroll 1
            for (int o = 0; o < HDP; o += 32) {
                uint32_t y[32];
                ap_ld32(y, 0, t_o + o);
                ap_wait_ld();
#pragma unroll
                for (int e = 0; e < 32; ++e) y[e] = seen > 0 ? __float_as_uint(__uint_as_float(y[e]) * inv) : 0u;
                if (poison && valid) {
                    const unsigned short *v = (const unsigned short *)a.v.data + kvh * a.v.head_stride;
                    for (int j = masked_from * AP_ROWS; j < seen; ++j)
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (o + e < a.hd) {
                                const unsigned short w = v[(long long)(k0 + j) * a.v.row_stride + o + e];
                                if (ap_nonfinite<T>(w) & 0x8000u) {
                                    T t;
                                    *(unsigned short *)&t = w;
                                    y[e] = __float_as_uint(__uint_as_float(y[e]) + (float)t);
                                }
                            }
                }
                if (valid) {
#pragma unroll
                    for (int e = 0; e < 32; e += 8)
                        if (o + e < a.hd) {
                            uint4 w;
                            w.x = ap_pack<T>(__uint_as_float(y[e]), __uint_as_float(y[e + 1]));
                            w.y = ap_pack<T>(__uint_as_float(y[e + 2]), __uint_as_float(y[e + 3]));
                            w.z = ap_pack<T>(__uint_as_float(y[e + 4]), __uint_as_float(y[e + 5]));
                            w.w = ap_pack<T>(__uint_as_float(y[e + 6]), __uint_as_float(y[e + 7]));
                            *(uint4 *)(out + o + e) = w;
                        }
                }
            }
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (warp == 9) {
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
    const cudaError_t e = cudaFuncSetAttribute(k_attn_prompt<T, HDP>, cudaFuncAttributeMaxDynamicSharedMemorySize, ApLayout<HDP>::SMEM);
    if (e != cudaSuccess) return e;
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
    const dim3 grid((unsigned)(n_q_rows / (2 * AP_ROWS) + std::min(n_seq, n_q_rows)), n_head);
    cudaStream_t st = (cudaStream_t)stream;
    cudaError_t ce;
    if (q->dtype == MDI_DTYPE_F16) ce = head_dim == 128 ? ap_launch<__half, 128>(mq, mk, mv, a, grid, st) : ap_launch<__half, 64>(mq, mk, mv, a, grid, st);
    else ce = head_dim == 128 ? ap_launch<__nv_bfloat16, 128>(mq, mk, mv, a, grid, st) : ap_launch<__nv_bfloat16, 64>(mq, mk, mv, a, grid, st);
    return op_cuda(who, ce);
}
