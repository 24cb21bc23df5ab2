// K8: attention with a window and first tokens, prompt form (sm_100a), and the host side of the windowed attention.
//
// The unit of work is two tiles of 128 query rows: the same rows of two query heads that share a key head (an even number
// of query heads for each key head), which then want the same key blocks, or else 256 rows of one head; one tile alone where the units would
// leave SMs without work.  A unit's key blocks of 64 are known from the rule: those of the first tokens and the window's, in one run
// (window::Blocks).  K and V stream through two rings of shared-memory stages that both tiles read; a tile issues no product for a
// block that none of its rows sees, a warp no exponential for a block that none of its sixteen rows sees, and only blocks on the edge of
// a row's window are compared number by number.
//
// One thread block per SM works through units until none is left, taking over those of thread blocks that have not started
// (clusterlaunchcontrol), so that a unit's first loads and scores run beside the epilogue of the one before.
// Roles (640 threads):
//   warps 0-15  softmax, eight warps per tile: a warp owns 16 query rows, a thread a quarter of two rows (16x256b fragments);
//               fp32 online softmax whose reference maximum moves only when a P would exceed 2^8, P written back over S, final O / l and lse
//   warp 16     producer: TMA loads of Q, then K and V blocks; K(g) and V(g - 1) complete one barrier.  V rows behind the sequence's
//               last key, which are not the caller's to keep finite, are set to zero here (0 * NaN would reach every row)
//   warps 17,18 UMMA issue, one warp per tile: S(n + NBUF - 1) = Q K^T is issued before O += P(n) V
//   warp 19     the next unit
// TMEM: tile t owns columns [256 t, 256 t + 256): S(n) at 64 (n mod NBUF), O behind the NBUF score buffers.
//
// Measured at D = 128 in a hot card's long run (from a cool start in brackets): 4608 tokens, 24 heads, 512 keys each way, 512 sinks that see all: 104 GFLOP of
// seen pairs in 124 us (114), 0.84 PFLOP/s; 8192 causal tokens, 32 heads on 8, window of 1024: 129 GFLOP in 174 us (152), 0.74 PFLOP/s.  Both tiles' work on a key
// block takes 1450 cycles, and 2 (8 x 32 + 4 x 64) = 1024 of these are the products' at the tensor cores' rate.  But with 64 columns a step of the scores' product is
// bounded by the shared memory that feeds it, 63 cycles for 32 of work, and 2 (8 x 63 + 4 x 64) = 1520 is all of the time.  So the softmax is not what bounds the
// loop: a share of the exponentials on the fma units gains nothing.  One product of 128 columns for two blocks' scores is not so bounded, but wants both buffers of
// scores, and then the softmax waits: 143 and 196 us.  Besides, a change of unit takes 4 us in each wave of units.
// The build for D = 64 keeps two registers a thread in local memory (4 bytes stored, 28 loaded).
// Every mbarrier wait is bounded; one that runs out is recorded (rapid3_window_status) and the thread block drains its copies and
// products, releases its TMEM and exits.
#include <float.h>
#include <math.h>
#include <stddef.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "window.cuh"

using namespace ptx;
using namespace window;

namespace {

constexpr int SOFTMAX_WARPS = 16, PRODUCER_WARP = 16, MMA_WARP0 = 17, NEXT_WARP = 19;
constexpr int NTHREADS = 32 * (SOFTMAX_WARPS + 4);
constexpr int SOFTMAX_REGS = 104, LIGHT_REGS = 64;       // registers a thread of the softmax warps, of the others: of 640 x 96
constexpr int TMEM_COLS = 512, TILE_COLS = 256;
constexpr int BLK_BYTES = 8192;                          // 64 rows x 64 channels
constexpr int QHALF_BYTES = 16384;                       // 128 rows x 64 channels
constexpr float GROWN_SUM = 256.0f, GROWN_LOG2 = 8.0f;   // when a row's reference maximum moves
constexpr float LOWEST = FLT_MAX;                        // reference maximum, times -c2, of a row that has seen nothing
constexpr int MAX_STAGES = 8, TAKE_AHEAD = 4;
constexpr int ABORT_EVERY = 32;
constexpr int UNIT_USERS = SOFTMAX_WARPS + 3;

__device__ int status_word;

struct Params {
    Rule w;
    Rows out;
    float* lse;
    int H, H_kv, group;
    int mode;                                            // 0: two heads, 1: 256 rows, 2: one tile
    int heads, row_tiles;                                // (sequence, head) pairs or pairs of heads; tiles of rows
    // The order: tiles of full rows, the longest, of all heads; then head by head, whose units share K and V in the L2 (with the heads
    // fastest 24 heads of 4608 tokens took 220 instead of 214 us, dense); the last rows first where these have the most keys.
    int full_tiles;
    bool last_first;
    float scale_log2;
};

template <int D>
struct Cfg {
    static constexpr int DH = D / 64;
    static constexpr int QTILE_BYTES = 128 * D * 2, KV_BYTES = 64 * D * 2;
    static constexpr int KS = D == 128 ? 4 : 8, VS = KS;
    static constexpr int DATA_BYTES = 2 * QTILE_BYTES + (KS + VS) * KV_BYTES;
    static constexpr int NBUF = D == 64 ? 3 : 2;
    static constexpr int O_COL = 64 * NBUF;
};

// A unit of work, written by the warp that takes it over: its index arithmetic is in no other role's way.
struct Unit {
    int n;                                               // key blocks; -1: no more units
    int b, hk, head[2], row0[2], rows, keys;             // row0 >= rows: nothing for that tile
    Blocks all;
    // of the unit's list of blocks a tile uses the first ones and those from `from` on, so many (0, 0: none)
    int first[2], from[2], count[2];
    // of a softmax warp's rows: see bounds_of
    int4 bounds[SOFTMAX_WARPS];
    int2 free[SOFTMAX_WARPS];
    __device__ __forceinline__ int tiles() const { return first[1] + count[1] > 0 ? 2 : 1; }
};

struct __align__(16) Ctl {
    uint4 taken;
    unsigned long long taken_full, near_end, tail_full;
    unsigned long long unit_full[2], unit_empty[2];
    unsigned long long q_full, q_empty;
    unsigned long long k_full[MAX_STAGES], k_empty[MAX_STAGES];   // k_full[g % KS]: group g = K(g) and V(g - 1) have landed
    unsigned long long v_empty[MAX_STAGES];
    unsigned long long s_full[2][3], p_full[2][3];
    unsigned long long pv_done[2][2], o_done[2], drain[2];
    uint32_t tmem_base;
    volatile int abort_flag;
    Unit unit[2];
};
template <int D>
constexpr size_t smem_bytes() { return (size_t)Cfg<D>::DATA_BYTES + sizeof(Ctl) + 1024; }

__device__ __forceinline__ Unit unit_of(const Params& p, int L) {
    Unit u;
    const int full = p.full_tiles * p.heads, tiles = L < full ? p.full_tiles : p.row_tiles - p.full_tiles;
    const int y = L < full ? L : L - full, x = y / tiles;
    int rt = y - x * tiles;
    if (p.last_first) rt = tiles - 1 - rt;
    if (L >= full) rt += p.full_tiles;
    if (p.mode == 0) {
        const int pairs = p.H / 2;
        u.b = x / pairs;
        u.head[0] = 2 * (x - u.b * pairs);
        u.head[1] = u.head[0] + 1;
        u.row0[0] = u.row0[1] = 128 * rt;
    } else {
        u.b = x / p.H;
        u.head[0] = u.head[1] = x - u.b * p.H;
        u.row0[0] = p.mode == 1 ? 256 * rt : 128 * rt;
        u.row0[1] = p.mode == 1 ? u.row0[0] + 128 : 1 << 30;      // (behind any row, and far from where int ends)
    }
    u.hk = u.head[0] / p.group;
    u.rows = p.w.rows(u.b);
    u.keys = p.w.keys(u.b);
    Blocks tile[2];
#pragma unroll
    for (int t = 0; t < 2; ++t)
        tile[t] = u.row0[t] < u.rows ? key_blocks(p.w, u.row0[t], min(u.row0[t] + 128, u.rows), u.rows, u.keys) : Blocks{0, 0, 0};
    u.all = tile[0].join(tile[1]);
    u.n = u.all.count();
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        u.first[t] = tile[t].first;
        u.from[t] = tile[t].from - u.all.from + u.all.first;
        u.count[t] = tile[t].to - tile[t].from;
    }
    return u;
}

// The first of a softmax warp's sixteen rows in its tile, and the tile.
__device__ __forceinline__ int row_of_warp(int warp) { return 32 * (warp & 3) + 16 * (warp >> 3); }
__device__ __forceinline__ int tile_of_warp(int warp) { return (warp >> 2) & 1; }

// Of the warp's rows: keys from none_from on are seen by none, nor, but for the first tokens, those below none_below; those from all_from
// up to all_to by all (so are the first tokens below all_to).  What lies between is compared.  free: the entries of the unit's list that all
// rows see whole, from where and how many.
__device__ __forceinline__ void bounds_of(const Rule& w, const Unit& u, int warp, int4& bounds, int2& free) {
    const int t = tile_of_warp(warp), row0 = (t ? u.row0[1] : u.row0[0]) + row_of_warp(warp), rows = u.rows, keys = u.keys;
    int none_from = 0, none_below = 0, all_from = 0, all_to = 0;
    if (row0 < rows) {
        const int p0 = row0 + keys - rows, p1 = min(row0 + 16, rows) - 1 + keys - rows;
        w.near(p0, keys, none_below, all_to);
        w.near(p1, keys, all_from, none_from);
        if (p0 < w.n_full && p1 >= 0) {                  // full rows among them
            none_from = keys;
            none_below = 0;
            int hi;
            w.seen(p1, keys, all_from, hi);
            if (p0 >= 0 && p1 < w.n_full) all_to = keys;
        }
    }
    bounds = make_int4(none_from, none_below, all_from, all_to);
    const int gap = u.all.from - u.all.first, from = max((all_from + 63) >> 6, u.all.from) - gap, to = min(all_to >> 6, u.all.to) - gap;
    free = make_int2(from, none_from > 0 && to > from ? to - from : 0);
}

__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// Maxima of a quad of lanes' two rows over one key block.
__device__ __forceinline__ void row_maxima(const uint32_t (&r)[32], float& lo, float& hi) {
    lo = hi = -INFINITY;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        lo = max3(lo, __uint_as_float(r[4 * k]), __uint_as_float(r[4 * k + 1]));
        hi = max3(hi, __uint_as_float(r[4 * k + 2]), __uint_as_float(r[4 * k + 3]));
    }
    lo = fmaxf(lo, __shfl_xor_sync(0xffffffffu, lo, 1));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, 1));
    lo = fmaxf(lo, __shfl_xor_sync(0xffffffffu, lo, 2));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, 2));
}

template <int D, int TYPE>
__global__ void __launch_bounds__(NTHREADS, 1)
window_kernel(const __grid_constant__ CUtensorMap tmq, const __grid_constant__ CUtensorMap tmk, const __grid_constant__ CUtensorMap tmv,
              const __grid_constant__ Params prm) {
    using C = Cfg<D>;
    constexpr int DH = C::DH, KS = C::KS, VS = C::VS, NBUF = C::NBUF, O_COL = C::O_COL, AHEAD = NBUF - 1;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw), pad = ((raw + 1023u) & ~1023u) - raw;
    uint8_t* smem = smem_raw + pad;
    const uint32_t sQ = raw + pad, sK = sQ + 2 * C::QTILE_BYTES, sV = sK + KS * C::KV_BYTES;
    Ctl* ctl = reinterpret_cast<Ctl*>(smem + C::DATA_BYTES);
    const int tid = threadIdx.x, lane = tid % 32;
    const int warp = __shfl_sync(0xffffffffu, tid / 32, 0);

    const uint32_t bQ = smem_u32(&ctl->q_full), bQE = smem_u32(&ctl->q_empty);
    const uint32_t bKF = smem_u32(&ctl->k_full[0]), bKE = smem_u32(&ctl->k_empty[0]), bVE = smem_u32(&ctl->v_empty[0]);
    const uint32_t bSF = smem_u32(&ctl->s_full[0][0]), bPF = smem_u32(&ctl->p_full[0][0]);   // [tile][buf]
    const uint32_t bPV = smem_u32(&ctl->pv_done[0][0]), bOD = smem_u32(&ctl->o_done[0]);
    const uint32_t bUF = smem_u32(&ctl->unit_full[0]), bUE = smem_u32(&ctl->unit_empty[0]);
    const uint32_t bNE = smem_u32(&ctl->near_end), bT = smem_u32(&ctl->taken_full), bTail = smem_u32(&ctl->tail_full);

    // ---------------------------------------------------------------- set-up
    if (warp == 0) {
        constexpr uint32_t at = offsetof(Ctl, taken_full) / 8, bars = offsetof(Ctl, tmem_base) / 8 - at;
        auto has = [&](uint32_t x, size_t member, int n) { return x + at - (uint32_t)(member / 8) < (uint32_t)n; };
#pragma unroll
        for (uint32_t x = lane; x < bars; x += 32) {
            uint32_t count = 1;
            if (has(x, offsetof(Ctl, unit_empty), 2)) count = UNIT_USERS;
            if (has(x, offsetof(Ctl, q_empty), 1) || has(x, offsetof(Ctl, k_empty), 2 * MAX_STAGES)) count = 2;   // both tiles pass a stage before it is refilled
            if (has(x, offsetof(Ctl, p_full), 6)) count = 8;                   // one arrival per softmax warp of the tile
            mbar_init(smem_u32(ctl) + 8 * (at + x), count);
        }
        if (lane == 0) ctl->abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == PRODUCER_WARP && lane < 3) prefetch_tmap(lane == 0 ? &tmq : lane == 1 ? &tmk : &tmv);
    if (warp == MMA_WARP0) {
        tmem_alloc(smem_u32(&ctl->tmem_base), TMEM_COLS);
        tmem_relinquish();
        tc_fence_before();
    }
    grid_dependency_wait();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = ctl->tmem_base;

    auto fail = [&]() {
        atomicExch(&status_word, RAPID3_ERR_TIMEOUT);
        ctl->abort_flag = 1;
    };
    // bounded wait that also gives up quickly once another role has failed
    auto wait = [&](uint32_t bar, uint32_t parity) -> bool {
        for (uint32_t it = 0; it < (1u << 22); ++it) {
            if (mbar_try_wait(bar, parity)) return true;
            if ((it & 15u) == 15u && ctl->abort_flag) return false;
        }
        fail();
        return false;
    };
    auto wait_warp = [&](uint32_t bar, uint32_t parity) -> bool { return __all_sync(0xffffffffu, wait(bar, parity)); };
    // one lane polls, where waits are long and the other lanes' polls would only take issue slots
    auto wait_lane0 = [&](uint32_t bar, uint32_t parity) -> bool {
        return __shfl_sync(0xffffffffu, (int)(lane != 0 || wait(bar, parity)), 0);
    };

    if (warp >= SOFTMAX_WARPS) reg_dec<LIGHT_REGS>();
    if (warp == NEXT_WARP) {
        // ------------------------------------------------------------ units
        int L = blockIdx.x;
        for (uint32_t i = 0;; ++i) {
            if (i > 1 && !wait_lane0(bUE + 8 * (i & 1), ((i >> 1) & 1) ^ 1)) break;
            Unit& to = ctl->unit[i & 1];
            if (L >= 0) {
                const Unit u = unit_of(prm, L);
                if (lane < SOFTMAX_WARPS) {
                    int4 bounds;
                    int2 free;
                    bounds_of(prm.w, u, lane, bounds, free);
                    to.bounds[lane] = bounds;
                    to.free[lane] = free;
                }
                if (lane == 0) {
                    to.n = u.n;
                    to.b = u.b;
                    to.hk = u.hk;
                    to.rows = u.rows;
                    to.keys = u.keys;
                    to.all = u.all;
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        to.head[t] = u.head[t];
                        to.row0[t] = u.row0[t];
                        to.first[t] = u.first[t];
                        to.from[t] = u.from[t];
                        to.count[t] = u.count[t];
                    }
                }
            } else if (lane == 0) {
                to.n = -1;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bUF + 8 * (i & 1));
            if (L < 0) break;
            if (!wait_lane0(bNE, i & 1)) break;          // the unit is nearly through
            if (lane == 0) {
                mbar_arrive_expect_tx(bT, 16);
                clc_try_cancel(smem_u32(&ctl->taken), bT);
            }
            __syncwarp();
            // no way out before the answer is here: it is written into this thread block's shared memory
            if (!__all_sync(0xffffffffu, mbar_wait(bT, i & 1))) {
                if (lane == 0) fail();
                break;
            }
            L = clc_taken(smem_u32(&ctl->taken));
        }
    } else if (warp == PRODUCER_WARP) {
        // ------------------------------------------------------------ producer, its warp converged
        // Groups and V blocks are numbered through all units: group gi of a unit is number G0 + gi (n + 1 of them, the last without
        // a K block), V block j number W0 + j.
        uint32_t G = 0, W0 = 0, n_q = 0, n_tail = 0;
        bool ok = true;
        for (uint32_t i = 0; ok; ++i) {
            if (!(ok = wait_lane0(bUF + 8 * (i & 1), (i >> 1) & 1))) break;
            const Unit& u = ctl->unit[i & 1];
            if (u.n < 0) break;
            if (u.n == 0 && lane == 0) mbar_arrive(bNE);
            // the last key's block, where rows behind it may hold anything
            const int tail = u.keys < prm.w.n_kv && (u.keys & 63) ? u.keys >> 6 : -1;
            for (int gi = 0; u.n > 0 && gi <= u.n; ++gi) {
                if (gi == max(u.n - TAKE_AHEAD, 0) && lane == 0) mbar_arrive(bNE);
                const uint32_t W = W0 + gi - 1, bar = bKF + 8 * (G % KS);
                // A group is issued once both ring stages it fills have been released.  The K stage's release also tells that both
                // MMA warps are past their wait on this barrier's previous phase, so it is awaited even without a K block.
                if (!(ok = wait_lane0(bKE + 8 * (G % KS), ((G / KS) & 1) ^ 1))) break;
                if (gi > 0 && !(ok = wait_lane0(bVE + 8 * (W % VS), ((W / VS) & 1) ^ 1))) break;
                const int kb = gi < u.n ? u.all.at(gi) : -1, vb = gi > 0 ? u.all.at(gi - 1) : -1;
                if (vb >= 0 && vb == tail) {
                    if (lane == 0) {
                        mbar_arrive_expect_tx(bTail, C::KV_BYTES);
#pragma unroll
                        for (int dh = 0; dh < DH; ++dh)
                            tma_load_4d(sV + (W % VS) * C::KV_BYTES + dh * BLK_BYTES, &tmv, bTail, dh * 64, vb * 64, u.hk, u.b);
                    }
                    __syncwarp();
                    if (!(ok = wait_lane0(bTail, n_tail++ & 1))) break;
                    uint8_t* v = smem + (sV - sQ) + (W % VS) * C::KV_BYTES;
                    const int first = u.keys & 63;       // a row of a half is 128 bytes; the swizzle moves bytes within it
                    for (int x = first * 8 + lane; x < 64 * 8; x += 32)
#pragma unroll
                        for (int dh = 0; dh < DH; ++dh) *reinterpret_cast<uint4*>(v + dh * BLK_BYTES + 16 * x) = make_uint4(0, 0, 0, 0);
                    fence_proxy_async_smem();
                    __syncwarp();
                }
                if (lane == 0) {
                    const bool v_here = vb >= 0 && vb != tail;
                    mbar_arrive_expect_tx(bar, (kb >= 0 ? C::KV_BYTES : 0) + (v_here ? C::KV_BYTES : 0));
#pragma unroll
                    for (int dh = 0; dh < DH; ++dh) {
                        if (kb >= 0) tma_load_4d(sK + (G % KS) * C::KV_BYTES + dh * BLK_BYTES, &tmk, bar, dh * 64, kb * 64, u.hk, u.b);
                        if (v_here) tma_load_4d(sV + (W % VS) * C::KV_BYTES + dh * BLK_BYTES, &tmv, bar, dh * 64, vb * 64, u.hk, u.b);
                    }
                }
                __syncwarp();
                ++G;
                if (gi == 0) {                           // the unit before has computed its last scores: its Q can go
                    if (n_q > 0 && !(ok = wait_lane0(bQE, (n_q - 1) & 1))) break;
                    if (lane == 0) {
                        const int tiles = u.tiles();       // (a first tile without blocks is loaded all the same)
                        mbar_arrive_expect_tx(bQ, tiles * C::QTILE_BYTES);
#pragma unroll
                        for (int a = 0; a < 4; ++a)
#pragma unroll
                            for (int dh = 0; dh < DH; ++dh)
                                if (a < 2 * tiles)
                                    tma_load_4d(sQ + (a >> 1) * C::QTILE_BYTES + dh * QHALF_BYTES + (a & 1) * BLK_BYTES, &tmq, bQ, dh * 64,
                                                u.row0[a >> 1] + 64 * (a & 1), u.head[a >> 1], u.b);
                    }
                    __syncwarp();
                    ++n_q;
                }
            }
            if (!ok) break;
            W0 += u.n;
            if (lane == 0) mbar_arrive(bUE + 8 * (i & 1));
        }
        if (ctl->abort_flag && lane == 0) {
            // drain: do not leave the thread block while copies may still land in its shared memory
            if (n_q > 0) mbar_wait(bQ, (n_q - 1) & 1, 1u << 20);
            if (n_tail > 0) mbar_wait(bTail, (n_tail - 1) & 1, 1u << 20);
            for (uint32_t x = G > KS ? G - KS : 0; x < G; ++x) mbar_wait(bKF + 8 * (x % KS), (x / KS) & 1, 1u << 20);
        }
        __syncwarp();
    } else if (warp >= MMA_WARP0) {
        // ------------------------------------------------------------ UMMA issue, one warp per tile
        // Both warps pass over every block, also those that their tile does not use, so that a stage is refilled only after both
        // are past it.  At D = 128 the elected lane runs the loop alone, without the votes that convergence costs.
        const int t = warp - MMA_WARP0;
        constexpr bool SOLO = D == 128;
        const bool leader = elect_one();
        auto mma_wait = [&](uint32_t bar, uint32_t parity) -> bool {
            if constexpr (SOLO) return wait(bar, parity);
            else return wait_warp(bar, parity);
        };
        if (!SOLO || leader) {
            const uint32_t tbase = tmem_base + t * TILE_COLS, tO = tbase + O_COL, qb = sQ + t * C::QTILE_BYTES;
            const uint32_t bSFt = bSF + 24 * t, bPFt = bPF + 24 * t;
            constexpr uint32_t idesc_qk = idesc16<TYPE>(128, 64, 0, 0), idesc_pv = idesc16<TYPE>(128, D, 0, 1);
            int n_qk = 0, n_pv = 0;                      // blocks of this tile issued so far, in all units
            uint32_t G0 = 0, W0 = 0, n_q = 0;
            bool ok = true;
            for (uint32_t i = 0; ok; ++i) {
                if (!(ok = mma_wait(bUF + 8 * (i & 1), (i >> 1) & 1))) break;
                const Unit& u = ctl->unit[i & 1];
                const int n_u = u.n, n_pv0 = n_pv;
                if (n_u < 0) break;
                const int use_first = u.first[t], use_from = u.from[t];
                const uint32_t use_count = u.count[t];
                auto used = [&](int j) { return (uint32_t)(j - use_from) < use_count || j < use_first; };
                auto k_step = [&](int j) -> bool {       // waits for group j, then issues S = Q K(j)^T
                    const uint32_t s = (G0 + j) % KS;
                    if (!mma_wait(bKF + 8 * s, ((G0 + j) / KS) & 1)) return false;
                    if (j >= n_u) {                      // the last group holds V(n_u - 1) only
                        if (leader) mbar_arrive(bKE + 8 * s);
                        return true;
                    }
                    if (used(j)) {
                        tc_fence_after();
                        const uint32_t tS = tbase + 64 * (n_qk % NBUF), kb = sK + s * C::KV_BYTES;
                        if (leader) {
#pragma unroll
                            for (int ks = 0; ks < D / 16; ++ks)
                                mma_ss(tS, smem_desc_sw128(qb + (ks / 4) * QHALF_BYTES + (ks % 4) * 32, 16, 1024),
                                       smem_desc_sw128(kb + (ks / 4) * BLK_BYTES + (ks % 4) * 32, 16, 1024), idesc_qk, ks > 0);
                            tc_commit(bKE + 8 * s);
                            tc_commit(bSFt + 8 * (n_qk % NBUF));
                        }
                        ++n_qk;
                    } else if (leader) {
                        mbar_arrive(bKE + 8 * s);
                    }
                    if (leader && j == n_u - 1) tc_commit(bQE);
                    if (!SOLO) __syncwarp();
                    return true;
                };
                if (n_u > 0) ok = mma_wait(bQ, n_q++ & 1);
                for (int j = 0; ok && n_u > 0 && j < AHEAD && j <= n_u; ++j) ok = k_step(j);
                for (int j = 0; ok && j < n_u; ++j) {
                    // S(n + NBUF - 1) reuses the buffer of P(n - 1); the MMAs of the issuing thread execute in issue order
                    if (j + AHEAD <= n_u && !(ok = k_step(j + AHEAD))) break;
                    const uint32_t s = (W0 + j) % VS;
                    if (used(j)) {
                        if (!(ok = mma_wait(bPFt + 8 * (n_pv % NBUF), (n_pv / NBUF) & 1))) break;
                        tc_fence_after();
                        const uint32_t tP = tbase + 64 * (n_pv % NBUF), vb = sV + s * C::KV_BYTES;
                        if (leader) {
                            // the first product of a unit overwrites O: that its P is there tells that every softmax warp of the
                            // tile has read the O of the unit before
#pragma unroll
                            for (int ks = 0; ks < 4; ++ks)
                                mma_ts(tO, tP + ks * 8, smem_desc_sw128(vb + ks * 2048, BLK_BYTES, 1024), idesc_pv, (n_pv > n_pv0 || ks > 0) ? 1u : 0u);
                            tc_commit(bVE + 8 * s);
                            tc_commit(bPV + 16 * t + 8 * (n_pv & 1));
                        }
                        ++n_pv;
                    } else if (leader) {
                        mbar_arrive(bVE + 8 * s);
                    }
                    if (!SOLO) __syncwarp();
                }
                if (!ok) break;
                if (leader) {
                    if (n_pv > n_pv0) tc_commit(bOD + 8 * t);
                    mbar_arrive(bUE + 8 * (i & 1));
                }
                if (!SOLO) __syncwarp();
                if (n_u > 0) G0 += n_u + 1;
                W0 += n_u;
            }
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------------ softmax, epilogue
        reg_inc<SOFTMAX_REGS>();
        const int t = tile_of_warp(warp);
        const int cg = lane & 3;                         // column pair within a group of eight
        const int row_w = row_of_warp(warp);
        const uint32_t lane_addr = tmem_base + ((uint32_t)row_w << 16) + t * TILE_COLS, tO = lane_addr + O_COL;
        const uint32_t bSFt = bSF + 24 * t, bPFt = bPF + 24 * t, bPVt = bPV + 16 * t;
        const float c2 = prm.scale_log2;
        int n = 0;                                       // blocks of this tile so far, in all units
        uint32_t n_o = 0;
        for (uint32_t i = 0;; ++i) {
            if (!wait_warp(bUF + 8 * (i & 1), (i >> 1) & 1)) break;
            const Unit& u = ctl->unit[i & 1];
            const int n_u = u.n;
            if (n_u < 0) break;
            // the loop keeps no more of them, it is short of registers
            const int free_from = u.free[warp].x;
            const uint32_t free_count = u.free[warp].y;
            float nm_lo = LOWEST, nm_hi = LOWEST;        // reference maxima of the two rows, times -c2
            float l0 = 0.f, l1 = 0.f, l2 = 0.f, l3 = 0.f;
            uint32_t r[32];
            const int n0 = n;
            bool seeded = false;
            // One block; FREE: all of the warp's rows see it whole.  (Two copies of the code: the one that most blocks take holds nothing else.)
            auto block = [&](int j, auto free) {
                    constexpr bool FREE = decltype(free)::value;
                    bool act = true, compare = false;
                    int key0 = 0;
                    if constexpr (!FREE) {
                        if ((uint32_t)(j - u.from[t]) >= (uint32_t)u.count[t] && j >= u.first[t]) return;      // none of the tile's rows sees it
                        const int4 bd = u.bounds[warp];
                        const int n_sink = prm.w.n_sink;
                        key0 = 64 * u.all.at(j);
                        act = key0 < bd.x && (key0 + 64 > bd.y || key0 < n_sink);
                        compare = key0 + 64 > bd.w || (key0 < bd.z && key0 + 64 > n_sink);
                    }
                    const int buf = n % NBUF;
                    const uint32_t tS = lane_addr + 64 * buf;
                    wait(bSFt + 8 * buf, (n / NBUF) & 1);
                    __syncwarp();
                    tc_fence_after();
                    uint32_t pk[16];
                    if (act) {
                        tmem_ld16x256_x8(tS, r);
                        tc_wait_ld();
                        if (!FREE && compare) {
                            // the keys of the block that the two rows see, as bits; the thread's columns 8 k + 2 cg + x at 8 k + x
                            uint32_t w0[2], w1[2];
                            const int row = u.row0[t] + row_w + (lane >> 2), rows = u.rows, keys = u.keys;
                            prm.w.seen_bits(row + keys - rows, row < rows ? keys : 0, key0, w0);
                            prm.w.seen_bits(row + 8 + keys - rows, row + 8 < rows ? keys : 0, key0, w1);
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                w0[h] >>= 2 * cg;
                                w1[h] >>= 2 * cg;
                            }
#pragma unroll
                            for (int k = 0; k < 8; ++k)
#pragma unroll
                                for (int x = 0; x < 2; ++x) {
                                    if (!(w0[k >> 2] >> (8 * (k & 3) + x) & 1u)) r[4 * k + x] = 0xff800000u;
                                    if (!(w1[k >> 2] >> (8 * (k & 3) + x) & 1u)) r[4 * k + 2 + x] = 0xff800000u;
                                }
                        }
                        // P = 2^(S c2 - m c2) with the reference maxima as they stand; only when a partial sum of eight exceeds 2^8 the
                        // maxima are taken, O and l rescaled and the pass repeated
                        float b0, b1, b2, b3;
                        if (!seeded) {
                            row_maxima(r, nm_lo, nm_hi);
                            nm_lo = fminf(nm_lo * -c2, LOWEST);
                            nm_hi = fminf(nm_hi * -c2, LOWEST);
                            seeded = true;
                        }
                        for (;;) {
                            b0 = b1 = b2 = b3 = 0.f;
#pragma unroll
                            for (int k = 0; k < 8; ++k) {
                                float x0, x1, x2, x3;
                                if (D == 64) {           // as packed pairs (dense, 24 heads of 4608 tokens: 188.5 -> 180.8 us; at D = 128 214.4 -> 215.8)
                                    const float2 lo = of_pair(fma2(pair_of(__uint_as_float(r[4 * k]), __uint_as_float(r[4 * k + 1])), pair_of(c2, c2), pair_of(nm_lo, nm_lo)));
                                    const float2 hi = of_pair(fma2(pair_of(__uint_as_float(r[4 * k + 2]), __uint_as_float(r[4 * k + 3])), pair_of(c2, c2), pair_of(nm_hi, nm_hi)));
                                    x0 = lo.x; x1 = lo.y; x2 = hi.x; x3 = hi.y;
                                } else {
                                    x0 = fmaf(__uint_as_float(r[4 * k]), c2, nm_lo); x1 = fmaf(__uint_as_float(r[4 * k + 1]), c2, nm_lo);
                                    x2 = fmaf(__uint_as_float(r[4 * k + 2]), c2, nm_hi); x3 = fmaf(__uint_as_float(r[4 * k + 3]), c2, nm_hi);
                                }
                                x0 = ex2(x0); x1 = ex2(x1); x2 = ex2(x2); x3 = ex2(x3);
                                add2(b0, b1, x0, x1);
                                add2(b2, b3, x2, x3);
                                pk[2 * k] = pack16<TYPE>(x0, x1);
                                pk[2 * k + 1] = pack16<TYPE>(x2, x3);
                            }
                            tmem_st16x128_x8(tS, pk);
                            if (!__any_sync(0xffffffffu, max3(b0, b1, fmaxf(b2, b3)) > GROWN_SUM)) break;
                            float mx_lo, mx_hi;
                            row_maxima(r, mx_lo, mx_hi);
                            mx_lo *= -c2; mx_hi *= -c2;
                            const bool g_lo = nm_lo - mx_lo > GROWN_LOG2, g_hi = nm_hi - mx_hi > GROWN_LOG2;
                            if (!__any_sync(0xffffffffu, g_lo || g_hi)) break;     // eight smaller P made the sum
                            tc_wait_st();                // nothing else orders the repeated pass's store of P behind this one's
                            if (n > n0) {
                                // O must be at rest: wait for P(n-1) V
                                wait(bPVt + 8 * ((n - 1) & 1), ((n - 1) >> 1) & 1);
                                __syncwarp();
                                tc_fence_after();
                                const float a_lo = g_lo ? ex2(mx_lo - nm_lo) : 1.f, a_hi = g_hi ? ex2(mx_hi - nm_hi) : 1.f;
                                l0 *= a_lo; l1 *= a_lo; l2 *= a_hi; l3 *= a_hi;
                                uint32_t o[16];
#pragma unroll
                                for (int ch = 0; ch < D / 32; ++ch) {
                                    tmem_ld16x256_x4(tO + ch * 32, o);
                                    tc_wait_ld();
#pragma unroll
                                    for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * ((e & 2) ? a_hi : a_lo));
                                    tmem_st16x256_x4(tO + ch * 32, o);
                                }
                            }
                            if (g_lo) nm_lo = mx_lo;
                            if (g_hi) nm_hi = mx_hi;
                        }
                        l0 += b0; l1 += b1; l2 += b2; l3 += b3;
                    } else {
#pragma unroll
                        for (int e = 0; e < 16; ++e) pk[e] = 0u;
                        tmem_st16x128_x8(tS, pk);
                    }
                    tc_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bPFt + 8 * buf);
                    ++n;
            };
            for (int j0 = 0; j0 < n_u;) {
                if (__any_sync(0xffffffffu, ctl->abort_flag)) break;
                const bool free = (uint32_t)(j0 - free_from) < free_count;
                const int j1 = min(j0 + ABORT_EVERY, free ? free_from + (int)free_count : j0 < free_from && free_count > 0 ? free_from : n_u);
                if (free) for (; j0 < j1; ++j0) block(j0, std::true_type());
                else for (; j0 < j1; ++j0) block(j0, std::false_type());
            }
            // epilogue: lse and 1 / l while the last product runs; O / l, 16 bytes a lane, four lanes a 64-byte piece of a row
            float s_lo = l0 + l1, s_hi = l2 + l3;
            s_lo += __shfl_xor_sync(0xffffffffu, s_lo, 1);
            s_hi += __shfl_xor_sync(0xffffffffu, s_hi, 1);
            s_lo += __shfl_xor_sync(0xffffffffu, s_lo, 2);
            s_hi += __shfl_xor_sync(0xffffffffu, s_hi, 2);
            const float inv_lo = s_lo > 0.f ? __fdividef(1.f, s_lo) : 0.f, inv_hi = s_hi > 0.f ? __fdividef(1.f, s_hi) : 0.f;   // a row that sees nothing: zeros
            const int b = u.b, head = u.head[t], row = u.row0[t] + row_w + (lane >> 2);
            const bool r0 = row < u.rows, r1 = row + 8 < u.rows;
            if (__any_sync(0xffffffffu, ctl->abort_flag)) break;
            if (prm.lse && cg == 0) {
                float* const to = prm.lse + ((long long)b * prm.H + head) * prm.w.n_q + row;
                if (r0) to[0] = s_lo > 0.f ? (__log2f(s_lo) - nm_lo) * 0.69314718055994531f : -INFINITY;
                if (r1) to[8] = s_hi > 0.f ? (__log2f(s_hi) - nm_hi) * 0.69314718055994531f : -INFINITY;
            }
            char* const o_lo = prm.out.row(b, head, row) + 16 * cg;
            char* const o_hi = o_lo + 16 * prm.out.n;
            if (n > n0) wait(bOD + 8 * t, n_o++ & 1);
            if (!__all_sync(0xffffffffu, !ctl->abort_flag)) break;
            tc_fence_after();
#pragma unroll
            for (int ch = 0; ch < D / 32; ch += 2) {
                uint32_t o[2][16];
                if (n > n0) {
                    tmem_ld16x256_x4(tO + ch * 32, o[0]);
                    tmem_ld16x256_x4(tO + ch * 32 + 32, o[1]);
                    tc_wait_ld();
                } else {
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[0][e] = o[1][e] = 0u;
                }
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    uint32_t w_lo[4], w_hi[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        w_lo[k] = pack16<TYPE>(__uint_as_float(o[x][4 * k]) * inv_lo, __uint_as_float(o[x][4 * k + 1]) * inv_lo);
                        w_hi[k] = pack16<TYPE>(__uint_as_float(o[x][4 * k + 2]) * inv_hi, __uint_as_float(o[x][4 * k + 3]) * inv_hi);
                    }
                    const uint4 v_lo = quad_transpose(w_lo[0], w_lo[1], w_lo[2], w_lo[3], cg);
                    const uint4 v_hi = quad_transpose(w_hi[0], w_hi[1], w_hi[2], w_hi[3], cg);
                    if (r0) *reinterpret_cast<uint4*>(o_lo + 64 * (ch + x)) = v_lo;
                    if (r1) *reinterpret_cast<uint4*>(o_hi + 64 * (ch + x)) = v_hi;
                    __syncwarp();
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bUE + 8 * (i & 1));
        }
    }

    // ---------------------------------------------------------------- teardown
    tc_fence_before();
    __syncthreads();
    if (warp >= MMA_WARP0 && warp < MMA_WARP0 + 2 && ctl->abort_flag) {
        // no UMMA of this warp may be in flight when the TMEM columns are released
        const uint32_t bD = smem_u32(&ctl->drain[warp - MMA_WARP0]);
        if (elect_one()) {
            tc_commit(bD);
            mbar_wait(bD, 0, 1u << 20);
        }
        __syncwarp();
    }
    __syncthreads();
    if (warp == MMA_WARP0) {
        tc_fence_after();
        tmem_dealloc(tmem_base, TMEM_COLS);
    }
}

// ------------------------------------------------------------------ host
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_fn() {
    static const EncodeTiledFn fn = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            f = nullptr;
        }
        return reinterpret_cast<EncodeTiledFn>(f);
    }();
    return fn;
}

cudaError_t static_init() {
    static std::atomic<uint64_t> done{0};                // devices, by bit
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t bit = 1ull << (dev & 63);
    if (dev < 64 && (done.load(std::memory_order_acquire) & bit)) return cudaSuccess;
    const void* kernels[] = {(const void*)window_kernel<128, RAPID3_BF16>, (const void*)window_kernel<128, RAPID3_F16>,
                             (const void*)window_kernel<64, RAPID3_BF16>, (const void*)window_kernel<64, RAPID3_F16>};
    for (int i = 0; i < 4; ++i) {
        if ((e = cudaFuncSetAttribute(kernels[i], cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(i < 2 ? smem_bytes<128>() : smem_bytes<64>()))) != cudaSuccess)
            return e;
        // the warps that take registers wait for them: a build that is launched with fewer would wait for good
        cudaFuncAttributes attr;
        if ((e = cudaFuncGetAttributes(&attr, kernels[i])) != cudaSuccess) return e;
        if (attr.numRegs * NTHREADS < 32 * (SOFTMAX_WARPS * SOFTMAX_REGS + 4 * LIGHT_REGS)) return cudaErrorInvalidKernelImage;
    }
    done.fetch_or(bit, std::memory_order_release);
    return cudaSuccess;
}

}  // namespace

namespace window {

int check(const rapid3_window* w) {
    if (!w) return RAPID3_ERR_INVALID_ARG;
    if (w->type != RAPID3_BF16 && w->type != RAPID3_F16) return w->type == RAPID3_F32 ? RAPID3_ERR_UNSUPPORTED : RAPID3_ERR_INVALID_ARG;
    if (w->D != 64 && w->D != 128) return RAPID3_ERR_UNSUPPORTED;
    if (w->B < 1 || w->H < 1 || w->H_kv < 1 || w->H % w->H_kv || w->n_q < 1 || w->n_kv < 1) return RAPID3_ERR_INVALID_ARG;
    if (w->n_q > MOST || w->n_kv > MOST || w->H > 65535 || (long long)w->B * w->H * ((w->n_q + 127ll) / 128) > (1 << 30) ||
        (long long)w->B * w->H_kv * ((w->n_kv + 127ll) / 128) > (1 << 30))
        return RAPID3_ERR_UNSUPPORTED;
    if (w->left < -1 || w->right < -1 || w->n_sink < 0 || w->n_full < 0) return RAPID3_ERR_INVALID_ARG;
    if (!(w->softmax_scale > 0.f) || !isfinite(w->softmax_scale * 1.4426950408889634f)) return RAPID3_ERR_INVALID_ARG;
    return RAPID3_OK;
}

int check_rows(const rapid3_window* w, const rapid3_rows* t, int heads, int n) {
    if (!t || !t->data || reinterpret_cast<uintptr_t>(t->data) % 16) return RAPID3_ERR_INVALID_ARG;
    const int64_t stride[3] = {t->stride_b, t->stride_h, t->stride_n};
    const int size[3] = {w->B, heads, n};
    for (int i = 0; i < 3; ++i) {
        if (size[i] == 1) continue;
        if (stride[i] < w->D || stride[i] % 8) return RAPID3_ERR_INVALID_ARG;
        if (stride[i] >= (1ll << 39)) return RAPID3_ERR_UNSUPPORTED;     // of a tensor map, in bytes
    }
    return RAPID3_OK;
}

Rule rule_of(const rapid3_window* w) {
    return {w->n_q, w->n_kv, std::min(w->left, MOST), std::min(w->right, MOST), std::min(w->n_sink, MOST), std::min(w->n_full, MOST),
            w->q_len, w->kv_len};
}

int tensor_map(const rapid3_window* w, const rapid3_rows* t, int heads, int n, CUtensorMap* map) {
    const EncodeTiledFn encode = encode_fn();
    if (!encode) return RAPID3_ERR_CUDA;
    const cuuint64_t row = 2 * (cuuint64_t)w->D;         // a dimension of one entry: any stride that is in order
    const cuuint64_t dims[4] = {(cuuint64_t)w->D, (cuuint64_t)n, (cuuint64_t)heads, (cuuint64_t)w->B};
    const cuuint64_t strides[3] = {n > 1 ? 2 * (cuuint64_t)t->stride_n : row, heads > 1 ? 2 * (cuuint64_t)t->stride_h : row,
                                   w->B > 1 ? 2 * (cuuint64_t)t->stride_b : row};
    const cuuint32_t box[4] = {64, 64, 1, 1}, one[4] = {1, 1, 1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, t->data, dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS ? RAPID3_OK : RAPID3_ERR_CUDA;
}

}  // namespace window

cudaError_t window_back_status(int* value, bool clear);  // k10_window_back.cu

extern "C" {

int rapid3_window_status(int* status) {
    if (!status) return RAPID3_ERR_INVALID_ARG;
    // Copies from and to symbols wait for the streams that the legacy default stream waits for, and no others.
    int forward = 0, back = 0;
    const int zero = 0;
    if (cudaDeviceSynchronize() != cudaSuccess || cudaMemcpyFromSymbol(&forward, status_word, sizeof(int)) != cudaSuccess ||
        window_back_status(&back, false) != cudaSuccess || (forward && cudaMemcpyToSymbol(status_word, &zero, sizeof(int)) != cudaSuccess) ||
        (back && window_back_status(&back, true) != cudaSuccess)) {
        cudaGetLastError();
        return RAPID3_ERR_CUDA;
    }
    *status = forward ? forward : back;
    return RAPID3_OK;
}

int rapid3_window_attn(const rapid3_window* w, const rapid3_rows* q, const rapid3_rows* k, const rapid3_rows* v, const rapid3_rows* out, float* lse,
                       void* stream) {
    int r = window::check(w);
    if (r || (r = window::check_rows(w, q, w->H, w->n_q)) || (r = window::check_rows(w, k, w->H_kv, w->n_kv)) ||
        (r = window::check_rows(w, v, w->H_kv, w->n_kv)) || (r = window::check_rows(w, out, w->H, w->n_q)))
        return r;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (window_rows_fit(w)) return launch_window_rows(w, q, k, v, out, lse, st) == cudaSuccess ? RAPID3_OK : RAPID3_ERR_CUDA;
    if (static_init() != cudaSuccess) {
        cudaGetLastError();
        return RAPID3_ERR_CUDA;
    }
    CUtensorMap tq, tk, tv;
    if ((r = window::tensor_map(w, q, w->H, w->n_q, &tq)) || (r = window::tensor_map(w, k, w->H_kv, w->n_kv, &tk)) ||
        (r = window::tensor_map(w, v, w->H_kv, w->n_kv, &tv)))
        return r;
    Params p;
    p.w = rule_of(w);
    p.out = rows_arg(out);
    p.lse = lse;
    p.H = w->H;
    p.H_kv = w->H_kv;
    p.group = w->H / w->H_kv;
    p.scale_log2 = w->softmax_scale * 1.4426950408889634f;
    p.last_first = w->left < 0 && w->right >= 0;
    const long long tiles = (long long)w->B * w->H * ((w->n_q + 127) / 128);
    p.mode = tiles <= SM_COUNT ? 2 : p.group % 2 == 0 ? 0 : 1;
    p.heads = w->B * w->H / (p.mode == 0 ? 2 : 1);
    p.row_tiles = p.mode == 1 ? (w->n_q + 255) / 256 : (w->n_q + 127) / 128;
    const long long full = std::min<long long>(w->n_q, w->n_full ? (long long)w->n_full + w->n_q - w->n_kv : 0);    // rows, of full sequences
    p.full_tiles = full > 0 ? (int)((full + (p.mode == 1 ? 255 : 127)) / (p.mode == 1 ? 256 : 128)) : 0;
    const bool bf = w->type == RAPID3_BF16;
    const auto kernel = w->D == 128 ? (bf ? window_kernel<128, RAPID3_BF16> : window_kernel<128, RAPID3_F16>)
                                    : (bf ? window_kernel<64, RAPID3_BF16> : window_kernel<64, RAPID3_F16>);
    return launch_kernel(kernel, dim3(p.heads * p.row_tiles), dim3(NTHREADS), w->D == 128 ? smem_bytes<128>() : smem_bytes<64>(), st, tq, tk, tv, p) == cudaSuccess
               ? RAPID3_OK : RAPID3_ERR_CUDA;
}

}  // extern "C"
