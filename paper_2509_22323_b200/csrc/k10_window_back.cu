// K10: gradients of attention with a window and first tokens (sm_100a).
//   P = exp(scale q k - lse) on the visible pairs, dP = dO V^T, dS = P (dP - delta), delta = sum over channels of dO O
//   dV = P^T dO,  dK = scale dS^T Q (summed over the query heads of a key head),  dQ = scale dS K
//
// No number is added to by two thread blocks, so the order of the sums is fixed and the same call gives the same bits: one kernel
// keeps a tile of 128 keys (or of 128 query rows) and streams blocks of 64 query rows (or keys) past it,
//   KEYS:   X1, X2 = K, V of the tile; Y1, Y2 = Q, dO of a block:  S^T = K Q^T, dP^T = V dO^T, then dV += P^T dO, dK += dS^T Q
//   else:   X1, X2 = Q, dO of the tile; Y1, Y2 = K, V of a block:  S = Q K^T,   dP = dO V^T,   then dQ += dS K
// seven products where five are the least (the scores and dP are computed twice); the other way, dQ by atomic additions of 32-bit partial
// sums to memory, costs 512 bytes of them for every row of every block and gives other bits on every call.
// P and dS go back to tensor memory, rounded to the tensors' type, as the first operand of the second products.
//
// Roles (576 threads): warps 0-15 the element work, eight warps per score buffer (blocks go to the two buffers by turns): a warp owns 16
// rows of the tile, a thread a quarter of two rows; warp 16 the producer (TMA; rows behind a sequence's last, which are not the caller's to
// keep finite, are set to zero); warp 17 the UMMA issue: S and dP of block n + 1 go out before the second products of block n.
// TMEM: 0 and D: the accumulators; 256 + 64 (n & 1): S; 384 + 64 (n & 1): dP.
// Every mbarrier wait is bounded, as in K8.
#include <math.h>
#include <stddef.h>

#include <algorithm>
#include <atomic>

#include "window.cuh"

using namespace ptx;
using namespace window;

namespace {

constexpr int WARPS = 16, PRODUCER_WARP = 16, MMA_WARP = 17, NTHREADS = 32 * (WARPS + 2);
constexpr int TMEM_COLS = 512, S_COL = 256, DP_COL = 384;
constexpr int BLK_BYTES = 8192, XHALF_BYTES = 16384;

__device__ int status_word;

struct Params {
    Rule w;
    Rows g1, g2;                 // KEYS: dK, dV; else dQ
    const float* lse2;           // [B][H][padded]: log sum exp in base 2; +inf: a row that has no P
    const float* delta;
    int padded;                  // query rows of a head in these, a multiple of 64
    int H, H_kv, group, tiles;   // tiles of a head
    float scale, scale_log2;
};

template <int D>
struct Cfg {
    static constexpr int DH = D / 64;
    static constexpr int XTILE_BYTES = 128 * D * 2, Y_BYTES = 64 * D * 2;
    static constexpr int STAT_BYTES = 512;                              // KEYS: lse2 and delta of the block's 64 rows
    static constexpr int STAGES = D == 128 ? 4 : 6;
    static constexpr int STAGE_BYTES = 2 * Y_BYTES;
    static constexpr int DATA_BYTES = 2 * XTILE_BYTES + STAGES * (STAGE_BYTES + STAT_BYTES);
};
constexpr int MAX_STAGES = 6;

struct __align__(16) Ctl {
    unsigned long long x_full, tail_full, full[MAX_STAGES], empty[MAX_STAGES], t_full[2], p_full[2], done, drain;
    uint32_t tmem_base;
    volatile int abort_flag;
};
template <int D>
constexpr size_t smem_bytes() { return (size_t)Cfg<D>::DATA_BYTES + sizeof(Ctl) + 1024; }

// The blocks of 64 query rows that see any of the keys [k0, k1).
__device__ __forceinline__ Blocks query_blocks(const Rule& w, int k0, int k1, int rows, int keys) {
    if (k0 >= keys) return {0, 0, 0};
    k1 = min(k1, keys);
    const int off = keys - rows;
    const int full = w.n_full == 0 ? 0 : min(max(w.n_full - off, 0), rows);   // behind the rows that see every key (before them there may be rows without a position)
    const int from = w.right < 0 ? 0 : min(max(k0 - w.right - off, 0), rows);
    const int to = w.left < 0 || k0 < w.n_sink ? rows : min(max(k1 + w.left - off, 0), rows);
    Blocks r;
    if (to <= from) {
        r.from = r.to = r.first = (full + 63) >> 6;
        return r;
    }
    r.from = from >> 6;
    r.to = (to + 63) >> 6;
    r.first = min((full + 63) >> 6, r.from);
    if (((full + 63) >> 6) > r.to) r.to = (full + 63) >> 6;             // (the window's rows lie among the full ones)
    return r;
}

template <int D, int TYPE, bool KEYS>
__global__ void __launch_bounds__(NTHREADS, 1)
window_back_kernel(const __grid_constant__ CUtensorMap tx1, const __grid_constant__ CUtensorMap tx2, const __grid_constant__ CUtensorMap ty1,
                   const __grid_constant__ CUtensorMap ty2, const __grid_constant__ Params prm) {
    using C = Cfg<D>;
    constexpr int DH = C::DH, STAGES = C::STAGES;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw), pad = ((raw + 1023u) & ~1023u) - raw;
    uint8_t* smem = smem_raw + pad;
    const uint32_t sX = raw + pad, sY = sX + 2 * C::XTILE_BYTES;
    const uint8_t* stats = smem + 2 * C::XTILE_BYTES + STAGES * C::STAGE_BYTES;
    Ctl* ctl = reinterpret_cast<Ctl*>(smem + C::DATA_BYTES);
    const int tid = threadIdx.x, lane = tid % 32;
    const int warp = __shfl_sync(0xffffffffu, tid / 32, 0);
    const uint32_t bX = smem_u32(&ctl->x_full), bTail = smem_u32(&ctl->tail_full), bF = smem_u32(&ctl->full[0]), bE = smem_u32(&ctl->empty[0]);
    const uint32_t bT = smem_u32(&ctl->t_full[0]), bP = smem_u32(&ctl->p_full[0]), bD = smem_u32(&ctl->done);

    if (warp == 0) {
        constexpr uint32_t bars = offsetof(Ctl, tmem_base) / 8;
        for (uint32_t x = lane; x < bars; x += 32) {
            uint32_t count = 1;
            if (x - (uint32_t)(offsetof(Ctl, p_full) / 8) < 2u) count = 8;             // one arrival per warp of the buffer
            mbar_init(smem_u32(ctl) + 8 * x, count);
        }
        if (lane == 0) ctl->abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == PRODUCER_WARP && lane < 4) prefetch_tmap(lane == 0 ? &tx1 : lane == 1 ? &tx2 : lane == 2 ? &ty1 : &ty2);
    if (warp == MMA_WARP) {
        tmem_alloc(smem_u32(&ctl->tmem_base), TMEM_COLS);
        tmem_relinquish();
        tc_fence_before();
    }
    grid_dependency_wait();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = ctl->tmem_base;

    // the tile: the longest ones first where the first rows or keys have the most work
    const int heads = KEYS ? prm.H_kv : prm.H;
    const int all_heads = gridDim.x / prm.tiles, tile = blockIdx.x / all_heads, at_head = blockIdx.x - tile * all_heads;
    const int b = at_head / heads, h = at_head - b * heads;
    const int rows = prm.w.rows(b), keys = prm.w.keys(b), off = keys - rows;
    const int first = 128 * tile, end = KEYS ? keys : rows;            // first row of the tile, of so many
    const Blocks blocks = first >= end ? Blocks{0, 0, 0} : KEYS ? query_blocks(prm.w, first, first + 128, rows, keys)
                                                                : key_blocks(prm.w, first, min(first + 128, rows), rows, keys);
    const int per_head = blocks.count(), n_items = KEYS ? prm.group * per_head : per_head;

    auto fail = [&]() {
        atomicExch(&status_word, RAPID3_ERR_TIMEOUT);
        ctl->abort_flag = 1;
    };
    auto wait = [&](uint32_t bar, uint32_t parity) -> bool {
        for (uint32_t it = 0; it < (1u << 22); ++it) {
            if (mbar_try_wait(bar, parity)) return true;
            if ((it & 15u) == 15u && ctl->abort_flag) return false;
        }
        fail();
        return false;
    };
    auto wait_lane0 = [&](uint32_t bar, uint32_t parity) -> bool {
        return __shfl_sync(0xffffffffu, (int)(lane != 0 || wait(bar, parity)), 0);
    };

    if (warp == PRODUCER_WARP) {
        int n = 0;
        uint32_t n_tail = 0;
        if (n_items > 0) {
            const int y_len = KEYS ? rows : keys, y_places = KEYS ? prm.w.n_q : prm.w.n_kv;
            const int tail = y_len < y_places && (y_len & 63) ? y_len >> 6 : -1;
            if (lane == 0) {
                mbar_arrive_expect_tx(bX, 2 * C::XTILE_BYTES);
#pragma unroll
                for (int a = 0; a < 2; ++a)
#pragma unroll
                    for (int dh = 0; dh < DH; ++dh) {
                        tma_load_4d(sX + dh * XHALF_BYTES + a * BLK_BYTES, &tx1, bX, dh * 64, first + 64 * a, h, b);
                        tma_load_4d(sX + C::XTILE_BYTES + dh * XHALF_BYTES + a * BLK_BYTES, &tx2, bX, dh * 64, first + 64 * a, h, b);
                    }
            }
            bool ok = true;
            for (int gh = 0; ok && gh < (KEYS ? prm.group : 1); ++gh)
                for (int j = 0; j < per_head; ++j, ++n) {
                    const int s = n % STAGES, block = blocks.at(j), yh = KEYS ? h * prm.group + gh : h / prm.group;
                    if (!(ok = wait_lane0(bE + 8 * s, ((n / STAGES) & 1) ^ 1))) break;
                    const uint32_t y = sY + s * C::STAGE_BYTES;
                    const bool mend = block == tail;
                    if (lane == 0) {
                        const uint32_t bar = mend ? bTail : bF + 8 * s;
                        mbar_arrive_expect_tx(bar, C::STAGE_BYTES + (KEYS ? C::STAT_BYTES : 0));
#pragma unroll
                        for (int dh = 0; dh < DH; ++dh) {
                            tma_load_4d(y + dh * BLK_BYTES, &ty1, bar, dh * 64, block * 64, yh, b);
                            tma_load_4d(y + C::Y_BYTES + dh * BLK_BYTES, &ty2, bar, dh * 64, block * 64, yh, b);
                        }
                        if (KEYS) {
                            const long long at = ((long long)b * prm.H + yh) * prm.padded + block * 64;
                            const uint32_t to = smem_u32(stats) + s * C::STAT_BYTES;
                            asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], 256, [%2];"
                                         ::"r"(to), "l"(prm.lse2 + at), "r"(bar) : "memory");
                            asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], 256, [%2];"
                                         ::"r"(to + 256), "l"(prm.delta + at), "r"(bar) : "memory");
                        }
                    }
                    __syncwarp();
                    if (mend) {
                        if (!(ok = wait_lane0(bTail, n_tail++ & 1))) break;
                        uint8_t* to = smem + (y - sX);
                        for (int z = (y_len & 63) * 8 + lane; z < 64 * 8; z += 32)
#pragma unroll
                            for (int dh = 0; dh < 2 * DH; ++dh) *reinterpret_cast<uint4*>(to + dh * BLK_BYTES + 16 * z) = make_uint4(0, 0, 0, 0);
                        fence_proxy_async_smem();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(bF + 8 * s);
                    }
                }
            if (ctl->abort_flag && lane == 0) {          // no copy may land after the thread block has left
                mbar_wait(bX, 0, 1u << 20);
                if (n_tail > 0) mbar_wait(bTail, (n_tail - 1) & 1, 1u << 20);
                for (int z = max(0, n - STAGES); z < n; ++z) mbar_wait(bF + 8 * (z % STAGES), (z / STAGES) & 1, 1u << 20);
            }
        }
        __syncwarp();
    } else if (warp == MMA_WARP) {
        if (elect_one() && n_items > 0) {
            constexpr uint32_t idesc1 = idesc16<TYPE>(128, 64, 0, 0), idesc2 = idesc16<TYPE>(128, D, 0, 1);
            bool ok = wait(bX, 0);
            auto first_products = [&](int n) -> bool {
                const int s = n % STAGES;
                if (!wait(bF + 8 * s, (n / STAGES) & 1)) return false;
                tc_fence_after();
                const uint32_t y = sY + s * C::STAGE_BYTES;
#pragma unroll
                for (int w = 0; w < 2; ++w)
#pragma unroll
                    for (int ks = 0; ks < D / 16; ++ks)
                        mma_ss(tmem_base + (w ? DP_COL : S_COL) + 64 * (n & 1),
                               smem_desc_sw128(sX + w * C::XTILE_BYTES + (ks / 4) * XHALF_BYTES + (ks % 4) * 32, 16, 1024),
                               smem_desc_sw128(y + w * C::Y_BYTES + (ks / 4) * BLK_BYTES + (ks % 4) * 32, 16, 1024), idesc1, ks > 0);
                tc_commit(bT + 8 * (n & 1));
                return true;
            };
            if (ok) ok = first_products(0);
            for (int n = 0; ok && n < n_items; ++n) {
                // S and dP of block n + 1 take the buffers of block n - 1, whose second products were issued before
                if (n + 1 < n_items && !(ok = first_products(n + 1))) break;
                if (!(ok = wait(bP + 8 * (n & 1), (n >> 1) & 1))) break;
                tc_fence_after();
                const int s = n % STAGES;
                const uint32_t y = sY + s * C::STAGE_BYTES;
                // KEYS: dK += dS^T Q, dV += P^T dO; else dQ += dS K
#pragma unroll
                for (int w = 0; w < (KEYS ? 2 : 1); ++w)
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks)
                        mma_ts(tmem_base + w * D, tmem_base + (w ? S_COL : DP_COL) + 64 * (n & 1) + ks * 8,
                               smem_desc_sw128(y + w * C::Y_BYTES + ks * 2048, BLK_BYTES, 1024), idesc2, (n > 0 || ks > 0) ? 1u : 0u);
                tc_commit(bE + 8 * s);
            }
            if (ok) tc_commit(bD);
        }
        __syncwarp();
    } else {
        const int set = warp >> 3, cg = lane & 3, row_w = 32 * (warp & 3) + 16 * ((warp >> 2) & 1);
        const uint32_t lane_addr = tmem_base + ((uint32_t)row_w << 16);
        const int row = first + row_w + (lane >> 2);     // and row + 8
        const float c2 = prm.scale_log2;
        // Where a row of the tile and a column of a block see one another: column in [lo, hi), or below `extra` (KEYS: the full rows;
        // else the first keys, below hi too).
        int lo[2], hi[2], extra = KEYS ? (prm.w.n_full == 0 ? 0 : prm.w.n_full - off) : prm.w.n_sink;
        float nl[2] = {0.f, 0.f}, dl[2] = {0.f, 0.f};
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = row + 8 * e;
            lo[e] = hi[e] = 0;
            if (r >= end) continue;
            if (KEYS) {
                lo[e] = prm.w.right < 0 ? 0 : max(r - prm.w.right - off, 0);
                hi[e] = prm.w.left < 0 || r < prm.w.n_sink ? rows : min(max(r + prm.w.left + 1 - off, 0), rows);
            } else {
                prm.w.seen(r + off, keys, lo[e], hi[e]);
                const long long at = ((long long)b * prm.H + h) * prm.padded + r;
                nl[e] = -__ldcg(prm.lse2 + at);
                dl[e] = __ldcg(prm.delta + at);
            }
        }
        // columns that all of the warp's rows see for certain: [all_from, all_to)
        const bool r0 = row < end, r1 = row + 8 < end;
        const int all_from = __reduce_max_sync(0xffffffffu, max(lo[0], lo[1]));
        const int all_to = __reduce_min_sync(0xffffffffu, min(r0 ? hi[0] : 0x7fffffff, r1 ? hi[1] : 0x7fffffff));
        for (int n = set; n < n_items; n += 2) {
            const int block = blocks.at(KEYS ? n % per_head : n), col0 = 64 * block;
            wait(bT + 8 * set, (n >> 1) & 1);
            if (KEYS) wait(bF + 8 * (n % STAGES), (n / STAGES) & 1);           // lse2 and delta of the block, read below
            if (__any_sync(0xffffffffu, ctl->abort_flag)) break;
            tc_fence_after();
            uint32_t s[32], d[32];
            tmem_ld16x256_x8(lane_addr + S_COL + 64 * set, s);
            tmem_ld16x256_x8(lane_addr + DP_COL + 64 * set, d);
            tc_wait_ld();
            const bool compare = col0 + 64 > all_to || col0 < all_from;
            const float* st = reinterpret_cast<const float*>(stats + (n % STAGES) * C::STAT_BYTES) + 2 * cg;
            uint32_t pp[16], pd[16];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                float nc[2] = {0.f, 0.f}, dc[2] = {0.f, 0.f};
                if (KEYS) {
                    const float2 a = *reinterpret_cast<const float2*>(st + 8 * k), bb = *reinterpret_cast<const float2*>(st + 64 + 8 * k);
                    nc[0] = -a.x; nc[1] = -a.y; dc[0] = bb.x; dc[1] = bb.y;
                }
                float p[4], ds[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int x2 = e & 1, r = e >> 1;
                    p[e] = ex2(fmaf(__uint_as_float(s[4 * k + e]), c2, KEYS ? nc[x2] : nl[r]));
                    ds[e] = p[e] * (__uint_as_float(d[4 * k + e]) - (KEYS ? dc[x2] : dl[r]));
                }
                if (compare) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int col = col0 + 8 * k + 2 * cg + (e & 1), r = e >> 1;
                        const bool seen = KEYS ? ((col >= lo[r] && col < hi[r]) || (col < extra && col >= -off)) : (col < hi[r] && (col >= lo[r] || col < extra));
                        if (!seen) p[e] = ds[e] = 0.f;
                    }
                }
                pp[2 * k] = pack16<TYPE>(p[0], p[1]);
                pp[2 * k + 1] = pack16<TYPE>(p[2], p[3]);
                pd[2 * k] = pack16<TYPE>(ds[0], ds[1]);
                pd[2 * k + 1] = pack16<TYPE>(ds[2], ds[3]);
            }
            if (KEYS) tmem_st16x128_x8(lane_addr + S_COL + 64 * set, pp);
            tmem_st16x128_x8(lane_addr + DP_COL + 64 * set, pd);
            tc_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bP + 8 * set);
        }
        if (n_items > 0) wait(bD, 0);
        if (__all_sync(0xffffffffu, !ctl->abort_flag)) {
            // epilogue: KEYS: half of the warps dK, half dV; else half of dQ's channels each
            tc_fence_after();
            constexpr int CH = KEYS ? D / 32 : D / 64;
            const Rows& to = KEYS && set ? prm.g2 : prm.g1;
            const float f = KEYS && set ? 1.f : prm.scale;
            const int ch0 = KEYS ? 0 : set * CH, col = KEYS ? set * D : 0;
            char* const o_lo = to.row(b, h, row) + 16 * cg + 64 * ch0;
            char* const o_hi = o_lo + 16 * to.n;
#pragma unroll
            for (int ch = 0; ch < CH; ++ch) {
                uint32_t o[16];
                if (n_items > 0) {
                    tmem_ld16x256_x4(lane_addr + col + (ch0 + ch) * 32, o);
                    tc_wait_ld();
                } else {
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[e] = 0u;
                }
                uint32_t w_lo[4], w_hi[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    w_lo[k] = pack16<TYPE>(__uint_as_float(o[4 * k]) * f, __uint_as_float(o[4 * k + 1]) * f);
                    w_hi[k] = pack16<TYPE>(__uint_as_float(o[4 * k + 2]) * f, __uint_as_float(o[4 * k + 3]) * f);
                }
                const uint4 v_lo = quad_transpose(w_lo[0], w_lo[1], w_lo[2], w_lo[3], cg);
                const uint4 v_hi = quad_transpose(w_hi[0], w_hi[1], w_hi[2], w_hi[3], cg);
                if (r0) *reinterpret_cast<uint4*>(o_lo + 64 * ch) = v_lo;
                if (r1) *reinterpret_cast<uint4*>(o_hi + 64 * ch) = v_hi;
            }
        }
    }

    tc_fence_before();
    __syncthreads();
    if (warp == MMA_WARP) {
        if (ctl->abort_flag) {                           // no UMMA may be in flight when the TMEM columns are released
            if (elect_one()) {
                tc_commit(smem_u32(&ctl->drain));
                mbar_wait(smem_u32(&ctl->drain), 0, 1u << 20);
            }
            __syncwarp();
        }
        tc_fence_after();
        tmem_dealloc(tmem_base, TMEM_COLS);
    }
}

// lse in base 2 and delta = sum dO O of every query row, padded to whole blocks with rows that have no P.  Bound by HBM: O and dO once.
template <int D, int TYPE>
__global__ void __launch_bounds__(256) row_stats_kernel(const Rule w, const Rows out, const Rows dout, const float* lse, float* lse2, float* delta,
                                                        int H, int padded) {
    constexpr int LPR = D / 8;                           // lanes of a row, 16 bytes each
    const int lane = threadIdx.x % LPR, i = blockIdx.x * (256 / LPR) + threadIdx.x / LPR, h = blockIdx.y % H, b = blockIdx.y / H;
    grid_dependency_wait();
    const bool there = i < w.rows(b);
    float sum = 0.f;
    if (there) {
        const uint4 o = __ldcg(reinterpret_cast<const uint4*>(out.row(b, h, i) + 16 * lane)), d = __ldcg(reinterpret_cast<const uint4*>(dout.row(b, h, i) + 16 * lane));
        const uint32_t ow[4] = {o.x, o.y, o.z, o.w}, dw[4] = {d.x, d.y, d.z, d.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 a = unpack16<TYPE>(ow[e]), c = unpack16<TYPE>(dw[e]);
            sum = fmaf(a.x, c.x, fmaf(a.y, c.y, sum));
        }
    }
#pragma unroll
    for (int x = 1; x < LPR; x <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
    grid_dependency_launch();
    if (lane == 0 && i < padded) {
        const float l = there ? __ldcg(lse + ((long long)b * H + h) * w.n_q + i) : -INFINITY;
        const long long at = ((long long)b * H + h) * padded + i;
        lse2[at] = l == -INFINITY ? INFINITY : l * 1.4426950408889634f;
        delta[at] = sum;
    }
}

template <int D, int TYPE>
cudaError_t static_init() {
    static std::atomic<uint64_t> done{0};                // devices, by bit
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t bit = 1ull << (dev & 63);
    if (dev < 64 && (done.load(std::memory_order_acquire) & bit)) return cudaSuccess;
    if ((e = cudaFuncSetAttribute(window_back_kernel<D, TYPE, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes<D>())) != cudaSuccess) return e;
    if ((e = cudaFuncSetAttribute(window_back_kernel<D, TYPE, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes<D>())) != cudaSuccess) return e;
    done.fetch_or(bit, std::memory_order_release);
    return cudaSuccess;
}

int padded_rows(const rapid3_window* w) { return (w->n_q + 63) / 64 * 64; }

template <int D, int TYPE>
int run(const rapid3_window* w, const rapid3_rows* q, const rapid3_rows* k, const rapid3_rows* v, const rapid3_rows* out, const float* lse,
        const rapid3_rows* dout, const rapid3_rows* dq, const rapid3_rows* dk, const rapid3_rows* dv, float* stats, cudaStream_t s) {
    if (static_init<D, TYPE>() != cudaSuccess) {
        cudaGetLastError();
        return RAPID3_ERR_CUDA;
    }
    CUtensorMap tq, tk, tv, td;
    int r;
    if ((r = tensor_map(w, q, w->H, w->n_q, &tq)) || (r = tensor_map(w, k, w->H_kv, w->n_kv, &tk)) || (r = tensor_map(w, v, w->H_kv, w->n_kv, &tv)) ||
        (r = tensor_map(w, dout, w->H, w->n_q, &td)))
        return r;
    Params p;
    p.w = rule_of(w);
    p.padded = padded_rows(w);
    float* const delta = stats + (size_t)w->B * w->H * p.padded;
    p.lse2 = stats;
    p.delta = delta;
    p.H = w->H;
    p.H_kv = w->H_kv;
    p.group = w->H / w->H_kv;
    p.scale = w->softmax_scale;
    p.scale_log2 = w->softmax_scale * 1.4426950408889634f;
    constexpr int PER = 256 / (D / 8);
    if (launch_kernel(row_stats_kernel<D, TYPE>, dim3((p.padded + PER - 1) / PER, w->B * w->H), dim3(256), 0, s, p.w, rows_arg(out), rows_arg(dout), lse,
                      stats, delta, w->H, p.padded) != cudaSuccess)
        return RAPID3_ERR_CUDA;
    p.g1 = rows_arg(dk);
    p.g2 = rows_arg(dv);
    p.tiles = (w->n_kv + 127) / 128;
    if (launch_kernel(window_back_kernel<D, TYPE, true>, dim3(w->B * w->H_kv * p.tiles), dim3(NTHREADS), smem_bytes<D>(), s, tk, tv, tq, td, p) != cudaSuccess)
        return RAPID3_ERR_CUDA;
    p.g1 = p.g2 = rows_arg(dq);
    p.tiles = (w->n_q + 127) / 128;
    if (launch_kernel(window_back_kernel<D, TYPE, false>, dim3(w->B * w->H * p.tiles), dim3(NTHREADS), smem_bytes<D>(), s, tq, td, tk, tv, p) != cudaSuccess)
        return RAPID3_ERR_CUDA;
    return RAPID3_OK;
}

}  // namespace

cudaError_t window_back_status(int* value) {
    cudaError_t e = cudaMemcpyFromSymbol(value, status_word, sizeof(int));
    const int zero = 0;
    return e != cudaSuccess ? e : cudaMemcpyToSymbol(status_word, &zero, sizeof(int));
}

extern "C" {

int64_t rapid3_window_workspace_bytes(const rapid3_window* w) {
    const int r = window::check(w);
    return r ? r : (int64_t)w->B * w->H * padded_rows(w) * 2 * sizeof(float);
}

int rapid3_window_attn_backward(const rapid3_window* w, const rapid3_rows* q, const rapid3_rows* k, const rapid3_rows* v, const rapid3_rows* out,
                                const float* lse, const rapid3_rows* dout, const rapid3_rows* dq, const rapid3_rows* dk, const rapid3_rows* dv,
                                void* workspace, int64_t workspace_bytes, void* stream) {
    int r = window::check(w);
    if (r) return r;
    for (const rapid3_rows* t : {q, out, dout, dq})
        if ((r = window::check_rows(w, t, w->H, w->n_q))) return r;
    for (const rapid3_rows* t : {k, v, dk, dv})
        if ((r = window::check_rows(w, t, w->H_kv, w->n_kv))) return r;
    if (!lse || !workspace || reinterpret_cast<uintptr_t>(workspace) % 16) return RAPID3_ERR_INVALID_ARG;
    if (workspace_bytes < rapid3_window_workspace_bytes(w)) return RAPID3_ERR_WORKSPACE;
    if ((long long)w->B * w->H > 65535) return RAPID3_ERR_UNSUPPORTED;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    float* stats = static_cast<float*>(workspace);
    const bool bf = w->type == RAPID3_BF16;
    return w->D == 128 ? (bf ? run<128, RAPID3_BF16>(w, q, k, v, out, lse, dout, dq, dk, dv, stats, s)
                             : run<128, RAPID3_F16>(w, q, k, v, out, lse, dout, dq, dk, dv, stats, s))
                       : (bf ? run<64, RAPID3_BF16>(w, q, k, v, out, lse, dout, dq, dk, dv, stats, s)
                             : run<64, RAPID3_F16>(w, q, k, v, out, lse, dout, dq, dk, dv, stats, s));
}

}  // extern "C"
