// K10: gradients of attention with a window and first tokens (sm_100a).
//   P = exp(scale q k - lse) on the visible pairs, dP = dO V^T, dS = P (dP - delta), delta = sum over channels of dO O
//   dV = P^T dO,  dK = scale dS^T Q (summed over the query heads of a key head),  dQ = scale dS K
//
// No number is added to by two thread blocks, so the order of the sums is fixed and the same call gives the same bits: a unit of work
// keeps a tile of 128 keys (or of 128 query rows) and streams blocks of 64 query rows (or keys) past it,
//   key unit:   X1, X2 = K, V of the tile; Y1, Y2 = Q, dO of a block:  S^T = K Q^T, dP^T = V dO^T, then dV += P^T dO, dK += dS^T Q
//   row unit:   X1, X2 = Q, dO of the tile; Y1, Y2 = K, V of a block:  S = Q K^T,   dP = dO V^T,   then dQ += dS K
// seven products where five are the least (the scores and dP are computed twice); the other way, dQ by atomic additions of 32-bit partial
// sums to memory, costs 512 bytes of them for every row of every block and gives other bits on every call.
// P and dS go back to tensor memory, rounded to the tensors' type, as the first operand of the second products.
//
// Both kinds of unit are one launch, the longest first: one thread block per SM works through them as in K8, and a unit's first loads and
// products run beside the last one's results on their way out.  Tiles of first tokens see every row, far more than the others: where they
// alone would keep a few SMs busy their blocks are shared out to several units, whose 32-bit results add_parts_kernel adds up.
//
// delta is made of the output that the caller has, which is rounded.  Of rows that see few keys, whose output is as large as a value, that
// shows: dq and dk of causal sequences were 1.5 to 1.8 times as far off as the rounding of the weights alone makes them (2.7 times at five
// tokens).  So tiles with rows that see fewer than EXACT_FROM keys (see few_tiles) have a launch of their own in front (`exact` row units), in which
// e = the sum of a row's dS, as they are before their rounding, is found: what delta was short of.
//     dQ = scale (sum dS K - e sum P K),   and delta + e is what the key units take
// A row that sees one key has dS = 0: its delta is marked by infinity, and both kinds of unit write zeros for it.
//
// Roles (640 threads): warps 0-15 the element work: a warp owns 16 rows of the tile, a thread a quarter of two rows; warp 16 the producer
// (TMA; rows behind a sequence's last, which are not the caller's to keep finite, are set to zero); warp 17 the UMMA issue; warp 18 the next unit.
//
// D = 64: eight warps a block, the blocks go to the two sets of eight by turns.  S and dP of block n + 2 go out before the second products of
// block n; tensor memory holds three buffers of 64 columns of S and 64 of dP behind the accumulators.
// D = 128: the first products are what bounds the kernel, not by the tensor cores' rate but by the shared memory that feeds them: with 64
// columns 16 x (128 + 64) numbers are read for 16 x 128 x 64 products, 48 cycles of the memory's 128 bytes for 32 cycles of work (measured: 63).
// So the blocks are 128 rows wide and the warps' two sets take their halves.  Tensor memory then holds one S and one dP beside the accumulators
// (0: dK or dQ, 128: dV, 256: S, 384: dP), and the element work goes in two steps: P from S, which stays in registers, so that the next
// block's S can follow at once; then dS from dP, and both, rounded, over the dP that the warp has read.  What is left in one chain is dS, the
// second products and the next block's dP (2000 cycles of a block's 3300); the element work takes as long, 350 instructions a warp at one in
// nine cycles.  Training pass of 4095 causal tokens, 32 heads on 8, window of 1024: blocks of 64 355 us, of 128 with P over S 349, so 335, and 356 with the
// launch for rows of few keys; 398 in a hot card's long run (one at a time: forward 89, row_stats_kernel 16, that launch 15, this one 267).  211 GFLOP of seen pairs.
// The exponential unit is not what it waits for: with a quarter or half of the powers on the fma units the 335 were 340 to 343.  The build of both kinds
// at D = 128 is short of registers: it keeps 56 bytes a thread in local memory (76 bytes of stores and 148 of loads in its code).
// P and dS in 16 bits cost 1.3 to 1.4 times the error of 32 bits; in fp16 dS beyond 65504 is infinite and below 2^-25 is 0.
// With lengths given the host does not know which tiles hold rows of few keys, and every row tile is in both launches, empty in one: the backward call of the
// case above 274 -> 294 us, of 2 x 1357 joint tokens, 24 heads, D = 64, 110 -> 121.
// Every mbarrier wait is bounded, as in K8.
#include <math.h>
#include <stddef.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "window.cuh"

using namespace ptx;
using namespace window;

namespace {

constexpr int WARPS = 16, PRODUCER_WARP = 16, MMA_WARP = 17, NEXT_WARP = 18, NTHREADS = 32 * (WARPS + 4);
constexpr int ELEMENT_REGS = 104, LIGHT_REGS = 64;       // registers a thread of the element warps, of the others: of 640 x 96
constexpr int TMEM_COLS = 512;
constexpr int BLK_BYTES = 8192, XHALF_BYTES = 16384;
constexpr int TAKE_AHEAD = 4, UNIT_USERS = WARPS + 2, ABORT_EVERY = 32;
constexpr int EXACT_FROM = 256;                          // at 128 keys a row and more the error is below 1.5 times that of the weights alone
constexpr int MAX_PARTS = 16, MAX_SLOTS = 2 * SM_COUNT;  // units of a shared-out tile; of all of them

__device__ int status_word;

struct Params {
    Rule w;
    Rows dq, dk, dv;
    const float* nlse;           // [B][H][padded]: minus log sum exp in base 2; -inf: a row that has no P
    float* ndelta;               // minus delta; +inf: a row that sees one key (exact row units bring it up to date)
    float* partial;              // [slot][128][2 D]
    int padded;                  // query rows of a head in these, a multiple of 128
    int H, H_kv, group;
    int key_tiles, row_tiles;    // of a head
    int sink_tiles, parts;       // the first key tiles, and how many units share one
    int full_tiles;              // the first row tiles
    int sink_units, key_units, full_units;   // where the kinds end in the order of the units: sink tiles, other key tiles, full row tiles, other row tiles
    bool last_first;             // the last rows have the most keys
    int few_tiles;               // the first row tiles, which may hold rows that see few keys
    int pass;                    // 0: all units; 1: tiles with such rows; 2: all others
    float scale, scale_log2;
};

template <int D>
struct Cfg {
    static constexpr int DH = D / 64;
    static constexpr bool WIDE = D == 128;
    static constexpr int WIDTH = WIDE ? 128 : 64;        // rows of a block
    static constexpr int XTILE_BYTES = 128 * D * 2, Y_BYTES = WIDTH * D * 2, YHALF_BYTES = WIDTH * 128;     // (a half: 64 channels)
    static constexpr int STAT_BYTES = 8 * WIDTH;         // key unit: nlse and ndelta of the block's rows
    static constexpr int NBUF = 3;
    static constexpr int S_COL = 2 * D, BUF_COLS = 128;                 // dP 64 columns behind S (WIDE: 128)
    static constexpr int STAGES = WIDE ? 2 : 6;
    static constexpr int STAGE_BYTES = 2 * Y_BYTES;
    static constexpr int DATA_BYTES = 2 * XTILE_BYTES + STAGES * (STAGE_BYTES + STAT_BYTES);
};
constexpr int MAX_STAGES = 6;

// A unit of work, written by the warp that takes it over.
struct Unit {
    int n;                       // its blocks, of all heads; -1: no more units
    int key;                     // a key unit
    int b, h, first, end;        // sequence, head (a key unit's: key head), first row of the tile, rows (keys) of the sequence
    int rows, keys;
    Blocks blocks;               // of one head
    int per_head, begin;         // a head's blocks; the first block of this part, through all heads
    int slot;                    // of a shared-out tile: where its result goes, else -1
    // Of an element warp's rows (eight groups of sixteen): columns in [x, y) and in [z, w) are seen by all rows; reach: by some at most from x up to y and
    // below z.
    int4 whole[8];
    int3 reach[8];
    int2 free[WARPS];            // of an element warp: the entries of a head's list whose 64 columns all rows see, from where and how many
};

struct __align__(16) Ctl {
    uint4 taken;
    unsigned long long taken_full, near_end, unit_full[2], unit_empty[2];
    unsigned long long x_full, x_empty, tail_full, full[MAX_STAGES], empty[MAX_STAGES], t_full[3], p_full[3], done, drained, drain, pair[8];
    uint32_t tmem_base;
    volatile int abort_flag;
    Unit unit[2];
    // exact: of a warp's rows, its columns' part of e.  By turns: a warp may be a unit ahead of the one it shares rows with, not two, since a Unit is
    // written again only when all have left the one before in its place.
    float short_of[2][WARPS][16];
};
template <int D>
constexpr size_t smem_bytes() { return (size_t)Cfg<D>::DATA_BYTES + sizeof(Ctl) + 1024; }

// Of a key: it is seen by the rows [lo, hi), and by the full ones.
__device__ __forceinline__ void rows_of_key(const Rule& w, int key, int rows, int off, int& lo, int& hi) {
    lo = w.right < 0 ? 0 : min(max(key - w.right - off, 0), rows);
    hi = w.left < 0 || key < w.n_sink ? rows : min(max(key + w.left + 1 - off, 0), rows);
}
// The full rows [lo, hi).
__device__ __forceinline__ void full_rows(const Rule& w, int rows, int off, int& lo, int& hi) {
    lo = min(max(-off, 0), rows);
    hi = w.n_full == 0 ? lo : min(max(w.n_full - off, lo), rows);
}
// The blocks of 64 query rows that see any of the keys [k0, k1), k1 <= keys.
__device__ __forceinline__ Blocks query_blocks(const Rule& w, int k0, int k1, int rows, int keys) {
    if (k0 >= k1) return {0, 0, 0};
    int from, to, x, full;
    rows_of_key(w, k0, rows, keys - rows, from, to);
    if (k0 >= w.n_sink) rows_of_key(w, k1 - 1, rows, keys - rows, x, to);
    full_rows(w, rows, keys - rows, x, full);
    if (full <= x) full = 0;
    const int full_blocks = (full + 63) >> 6;
    Blocks r;
    if (to <= from) {
        r.from = r.to = r.first = full_blocks;
        return r;
    }
    r.from = from >> 6;
    r.to = max((to + 63) >> 6, full_blocks);
    r.first = min(full_blocks, r.from);
    return r;
}

// Of sixteen rows of a tile, see Unit::whole and reach.
__device__ __forceinline__ void bounds_of(const Rule& w, const Unit& u, int group, int4& whole, int3& reach) {
    const int r0 = u.first + 16 * group, r1 = min(r0 + 16, u.end) - 1, off = u.keys - u.rows;
    whole = make_int4(0, 0, 0, 0);
    reach = make_int3(0, 0, 0);
    if (r0 > r1) return;
    if (u.key) {
        const bool lone = r0 == r1;                      // every block is looked at for rows that see this key alone, see `mark`
        int lo, hi, from, to;
        rows_of_key(w, r0, u.rows, off, from, hi);       // from: the least; hi: the least unless the row is a first token
        rows_of_key(w, r1, u.rows, off, lo, to);
        if (r0 < w.n_sink) {
            to = u.rows;
            int x;
            if (r1 >= w.n_sink) rows_of_key(w, w.n_sink, u.rows, off, x, hi);
        }
        int full_lo, full_hi;
        full_rows(w, u.rows, off, full_lo, full_hi);
        whole = lone ? make_int4(0, 0, 0, 0) : make_int4(lo, hi, full_lo, full_hi);
        reach = make_int3(from, to, full_hi);
    } else {
        const int p0 = r0 + off, p1 = r1 + off;
        int lo, hi, from, to;
        w.near(p0, u.keys, from, hi);
        w.near(p1, u.keys, lo, to);
        if (p0 < w.n_full && p1 >= 0) {                  // full rows among them
            int x;
            from = 0;
            to = u.keys;
            w.seen(p1, u.keys, lo, x);
            if (p0 >= 0 && p1 < w.n_full) hi = u.keys;
        }
        whole = make_int4(lo, hi, 0, min(w.n_sink, hi));
        reach = make_int3(from, to, min(w.n_sink, to));
    }
}

// Unit::free, from the first of the two ranges.
__device__ __forceinline__ int2 free_of(const Unit& u, const int4& whole, int set, bool wide) {
    const int shift = wide ? 7 : 6, add = wide ? 64 * set : 0, from = max((whole.x - add + (1 << shift) - 1) >> shift, u.blocks.from);
    const int to = min(((whole.y - add - 64) >> shift) + 1, u.blocks.to), gap = u.blocks.from - u.blocks.first;
    return make_int2(from - gap, max(to - from, 0));
}
// Blocks of 64 as blocks of 128.
__device__ __forceinline__ Blocks doubled(const Blocks& b) {
    Blocks r;
    r.from = b.from >> 1;
    r.to = (b.to + 1) >> 1;
    r.first = min((b.first + 1) >> 1, r.from);
    return r;
}

__device__ __forceinline__ Unit unit_of(const Params& p, int B, int L, bool wide) {
    Unit u;
    u.key = p.pass != 1 && L < p.key_units;
    u.slot = -1;
    const int heads = B * (u.key ? p.H_kv : p.H);
    int part = 0, parts = 1, x, tile;
    if (p.pass == 1) {
        x = L / p.few_tiles;
        tile = L - x * p.few_tiles;
    } else if (L < p.sink_units) {
        parts = p.parts;
        x = L / parts;
        part = L - x * parts;
        if (parts > 1) u.slot = L;
        tile = x / heads;                                // tiles of first tokens: of all heads side by side
        x -= tile * heads;
    } else {
        const bool full = !u.key && L < p.full_units;
        const int tiles = u.key ? p.key_tiles - p.sink_tiles : full ? p.full_tiles : p.row_tiles - p.full_tiles;
        const int y = L - (u.key ? p.sink_units : full ? p.key_units : p.full_units);
        x = y / tiles;                                   // head by head, whose units share what they stream in the L2
        tile = y - x * tiles;
        if (!u.key && p.last_first) tile = tiles - 1 - tile;
        tile += u.key ? p.sink_tiles : full ? 0 : p.full_tiles;
    }
    const int per = u.key ? p.H_kv : p.H;
    u.b = x / per;
    u.h = x - u.b * per;
    u.rows = p.w.rows(u.b);
    u.keys = p.w.keys(u.b);
    u.first = 128 * tile;
    u.end = u.key ? u.keys : u.rows;
    if (!u.key && p.pass != 0) {
        const int off = u.keys - u.rows;
        // each tile in its pass (the rows of a tile that see the least are its first or its last)
        if (u.first < u.end && (min(p.w.count(u.first + off, u.keys), p.w.count(min(u.first + 128, u.end) - 1 + off, u.keys)) < EXACT_FROM) != (p.pass == 1))
            u.end = u.first;
    }
    const int last = min(u.first + 128, u.end);
    u.blocks = u.first >= last ? Blocks{0, 0, 0} : u.key ? query_blocks(p.w, u.first, last, u.rows, u.keys)
                                                         : key_blocks(p.w, u.first, last, u.rows, u.keys);
    if (wide && u.blocks.count() > 0) u.blocks = doubled(u.blocks);
    u.per_head = u.blocks.count();
    const int n = u.key ? p.group * u.per_head : u.per_head;
    u.begin = (int)((long long)n * part / parts);
    u.n = (int)((long long)n * (part + 1) / parts) - u.begin;
    return u;
}

// The blocks of a unit one after the other: of which head of the group, and which.
struct Walk {
    int head, j;
    __device__ __forceinline__ Walk(const Unit& u) {
        head = u.per_head > 0 ? u.begin / u.per_head : 0;
        j = u.begin - head * u.per_head;
    }
    __device__ __forceinline__ void next(int per_head) {
        if (++j == per_head) {
            j = 0;
            ++head;
        }
    }
};

// EXACT: the build of pass 1, for exact row units alone.
template <int D, int TYPE, bool EXACT>
__global__ void __launch_bounds__(NTHREADS, 1)
window_back_kernel(const __grid_constant__ CUtensorMap tq, const __grid_constant__ CUtensorMap tk, const __grid_constant__ CUtensorMap tv,
                   const __grid_constant__ CUtensorMap td, const __grid_constant__ Params prm, int B) {
    using C = Cfg<D>;
    constexpr int DH = C::DH, STAGES = C::STAGES, NBUF = C::NBUF, WIDTH = C::WIDTH;
    constexpr bool WIDE = C::WIDE;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw), pad = ((raw + 1023u) & ~1023u) - raw;
    uint8_t* smem = smem_raw + pad;
    const uint32_t sX = raw + pad, sY = sX + 2 * C::XTILE_BYTES;
    const uint8_t* stats = smem + 2 * C::XTILE_BYTES + STAGES * C::STAGE_BYTES;
    Ctl* ctl = reinterpret_cast<Ctl*>(smem + C::DATA_BYTES);
    const int tid = threadIdx.x, lane = tid % 32;
    const int warp = __shfl_sync(0xffffffffu, tid / 32, 0);
    const uint32_t bX = smem_u32(&ctl->x_full), bXE = smem_u32(&ctl->x_empty), bTail = smem_u32(&ctl->tail_full);
    const uint32_t bF = smem_u32(&ctl->full[0]), bE = smem_u32(&ctl->empty[0]), bT = smem_u32(&ctl->t_full[0]), bP = smem_u32(&ctl->p_full[0]);
    const uint32_t bD = smem_u32(&ctl->done), bDE = smem_u32(&ctl->drained);
    const uint32_t bPair = smem_u32(&ctl->pair[0]);
    const uint32_t bUF = smem_u32(&ctl->unit_full[0]), bUE = smem_u32(&ctl->unit_empty[0]), bNE = smem_u32(&ctl->near_end), bTk = smem_u32(&ctl->taken_full);

    if (warp == 0) {
        constexpr uint32_t at = offsetof(Ctl, taken_full) / 8, bars = offsetof(Ctl, tmem_base) / 8 - at;
        auto has = [&](uint32_t x, size_t member, int n) { return x + at - (uint32_t)(member / 8) < (uint32_t)n; };
        for (uint32_t x = lane; x < bars; x += 32) {
            uint32_t count = 1;
            if (has(x, offsetof(Ctl, unit_empty), 2)) count = UNIT_USERS;
            if (has(x, offsetof(Ctl, p_full), 3)) count = WIDE ? WARPS : 8;     // one arrival per warp that works on the buffer
            if (has(x, offsetof(Ctl, drained), 1)) count = WARPS;
            if (has(x, offsetof(Ctl, pair), 8)) count = 2;                      // both sets' warps of the rows
            mbar_init(smem_u32(ctl) + 8 * (at + x), count);
        }
        if (lane == 0) ctl->abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == PRODUCER_WARP && lane < 4) prefetch_tmap(lane == 0 ? &tq : lane == 1 ? &tk : lane == 2 ? &tv : &td);
    if (warp == MMA_WARP) {
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

    if (warp >= WARPS) reg_dec<LIGHT_REGS>();
    if (warp == NEXT_WARP) {
        int L = blockIdx.x;
        for (uint32_t i = 0;; ++i) {
            if (i > 1 && !wait_lane0(bUE + 8 * (i & 1), ((i >> 1) & 1) ^ 1)) break;
            Unit& to = ctl->unit[i & 1];
            if (L >= 0) {
                const Unit u = unit_of(prm, B, L, C::WIDE);
                if (lane < 8) {
                    int4 whole;
                    int3 reach;
                    bounds_of(prm.w, u, lane, whole, reach);
                    to.whole[lane] = whole;
                    to.reach[lane] = reach;
#pragma unroll
                    for (int set = 0; set < 2; ++set) to.free[2 * lane + set] = free_of(u, whole, set, C::WIDE);
                }
                if (lane == 0) {
                    to.n = u.n; to.key = u.key; to.b = u.b; to.h = u.h;
                    to.first = u.first; to.end = u.end; to.rows = u.rows; to.keys = u.keys;
                    to.blocks = u.blocks; to.per_head = u.per_head; to.begin = u.begin; to.slot = u.slot;
                }
            } else if (lane == 0) {
                to.n = -1;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bUF + 8 * (i & 1));
            if (L < 0) break;
            if (!wait_lane0(bNE, i & 1)) break;          // the unit is nearly through
            if (lane == 0) {
                mbar_arrive_expect_tx(bTk, 16);
                clc_try_cancel(smem_u32(&ctl->taken), bTk);
            }
            __syncwarp();
            // no way out before the answer is here: it is written into this thread block's shared memory
            if (!__all_sync(0xffffffffu, mbar_wait(bTk, i & 1))) {
                if (lane == 0) fail();
                break;
            }
            L = clc_taken(smem_u32(&ctl->taken));
        }
    } else if (warp == PRODUCER_WARP) {
        uint32_t N = 0, n_x = 0, n_tail = 0;             // blocks, tiles and mended blocks so far, in all units
        bool ok = true;
        for (uint32_t i = 0; ok; ++i) {
            if (!(ok = wait_lane0(bUF + 8 * (i & 1), (i >> 1) & 1))) break;
            const Unit& u = ctl->unit[i & 1];
            const int n = u.n, per_head = u.per_head, b = u.b, h = u.h;
            if (n < 0) break;
            const bool key = u.key;
            const Blocks blocks = u.blocks;
            const CUtensorMap* const x1 = key ? &tk : &tq, * const x2 = key ? &tv : &td, * const y1 = key ? &tq : &tk, * const y2 = key ? &td : &tv;
            const int y_len = key ? u.rows : u.keys, y_places = key ? prm.w.n_q : prm.w.n_kv;
            const int tail = y_len < y_places && y_len % WIDTH ? y_len / WIDTH : -1;
            if (n == 0 && lane == 0) mbar_arrive(bNE);
            Walk at(u);
            for (int j = 0; j < n; ++j, ++N, at.next(per_head)) {
                if (j == max(n - TAKE_AHEAD, 0) && lane == 0) mbar_arrive(bNE);
                if (j == 0) {                            // the unit before has computed its last scores: its tile can go
                    if (n_x > 0 && !(ok = wait_lane0(bXE, (n_x - 1) & 1))) break;
                    if (lane == 0) {
                        const int first = u.first;
                        mbar_arrive_expect_tx(bX, 2 * C::XTILE_BYTES);
#pragma unroll
                        for (int a = 0; a < 2; ++a)
#pragma unroll
                            for (int dh = 0; dh < DH; ++dh) {
                                tma_load_4d(sX + dh * XHALF_BYTES + a * BLK_BYTES, x1, bX, dh * 64, first + 64 * a, h, b);
                                tma_load_4d(sX + C::XTILE_BYTES + dh * XHALF_BYTES + a * BLK_BYTES, x2, bX, dh * 64, first + 64 * a, h, b);
                            }
                    }
                    ++n_x;
                }
                const uint32_t s = N % STAGES;
                const int block = blocks.at(at.j), yh = key ? h * prm.group + at.head : h / prm.group;
                // WIDE: Y1 and Y2 have stages and barriers of their own
                constexpr int LOADS = WIDE ? 2 : 1;
#pragma unroll
                for (int x = 0; x < LOADS; ++x) {
                    if (!(ok = wait_lane0(bE + 8 * (x * STAGES + s), ((N / STAGES) & 1) ^ 1))) break;
                    const uint32_t y = sY + s * C::STAGE_BYTES;
                    const bool mend = block == tail;
                    const uint32_t full = bF + 8 * (x * STAGES + s);
                    if (lane == 0) {
                        const uint32_t bar = mend ? bTail : full;
                        mbar_arrive_expect_tx(bar, C::STAGE_BYTES / LOADS + (key && x == 0 ? C::STAT_BYTES : 0));
#pragma unroll
                        for (int dh = 0; dh < DH; ++dh)
#pragma unroll
                            for (int a = 0; a < WIDTH / 64; ++a) {
                                const int row = block * WIDTH + 64 * a;
                                if (!WIDE || x == 0) tma_load_4d(y + dh * C::YHALF_BYTES + a * BLK_BYTES, y1, bar, dh * 64, row, yh, b);
                                if (!WIDE || x == 1) tma_load_4d(y + C::Y_BYTES + dh * C::YHALF_BYTES + a * BLK_BYTES, y2, bar, dh * 64, row, yh, b);
                            }
                        if (key && x == 0) {             // (with Y1, whose stage stays until dS is there)
                            const long long from = ((long long)b * prm.H + yh) * prm.padded + block * WIDTH;
                            const uint32_t to = smem_u32(stats) + s * C::STAT_BYTES;
                            asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %3, [%2];"
                                             ::"r"(to), "l"(prm.nlse + from), "r"(bar), "n"(4 * WIDTH) : "memory");
                            asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %3, [%2];"
                                             ::"r"(to + 4 * WIDTH), "l"(prm.ndelta + from), "r"(bar), "n"(4 * WIDTH) : "memory");
                        }
                    }
                    __syncwarp();
                    if (mend) {
                        if (!(ok = wait_lane0(bTail, n_tail++ & 1))) break;
                        uint8_t* to = smem + (y - sX) + (x == 1 ? C::Y_BYTES : 0);       // a row of a half is 128 bytes; the swizzle moves bytes within it
                        for (int z = y_len % WIDTH * 8 + lane; z < WIDTH * 8; z += 32)
#pragma unroll
                            for (int dh = 0; dh < 2 * DH / LOADS; ++dh) *reinterpret_cast<uint4*>(to + dh * C::YHALF_BYTES + 16 * z) = make_uint4(0, 0, 0, 0);
                        fence_proxy_async_smem();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(full);
                    }
                }
                if (!ok) break;
            }
            if (!ok) break;
            if (lane == 0) mbar_arrive(bUE + 8 * (i & 1));
        }
        if (ctl->abort_flag && lane == 0) {              // no copy may land after the thread block has left
            if (n_x > 0) mbar_wait(bX, (n_x - 1) & 1, 1u << 20);
            if (n_tail > 0) mbar_wait(bTail, (n_tail - 1) & 1, 1u << 20);
            for (uint32_t z = N > STAGES ? N - STAGES : 0; z < N; ++z)
                for (int x = 0; x < (WIDE ? 2 : 1); ++x) mbar_wait(bF + 8 * (x * STAGES + z % STAGES), (z / STAGES) & 1, 1u << 20);
            // (of a block whose first load alone was issued)
            if (WIDE) mbar_wait(bF + 8 * (N % STAGES), (N / STAGES) & 1, 1u << 12);
        }
        __syncwarp();
    } else if (warp == MMA_WARP) {
        if (elect_one()) {
            constexpr uint32_t idesc1 = idesc16<TYPE>(128, WIDTH, 0, 0), idesc2 = idesc16<TYPE>(128, D, 0, 1);
            uint32_t N = 0, n_x = 0;
            bool ok = true;
            for (uint32_t i = 0; ok; ++i) {
                if (!(ok = wait(bUF + 8 * (i & 1), (i >> 1) & 1))) break;
                const int n = ctl->unit[i & 1].n;
                const bool key = !EXACT && ctl->unit[i & 1].key;
                if (n < 0) break;
                if constexpr (WIDE) {
                    // w = 0: S from Y1, 1: dP from Y2
                    auto first_product = [&](int j, int w) -> bool {
                        const uint32_t M = N + j, s = M % STAGES;
                        if (!wait(bF + 8 * (w * STAGES + s), (M / STAGES) & 1)) return false;
                        tc_fence_after();
                        const uint32_t y = sY + s * C::STAGE_BYTES + w * C::Y_BYTES;
#pragma unroll
                        for (int ks = 0; ks < D / 16; ++ks)
                            mma_ss(tmem_base + C::S_COL + 128 * w, smem_desc_sw128(sX + w * C::XTILE_BYTES + (ks / 4) * XHALF_BYTES + (ks % 4) * 32, 16, 1024),
                                   smem_desc_sw128(y + (ks / 4) * C::YHALF_BYTES + (ks % 4) * 32, 16, 1024), idesc1, ks > 0);
                        tc_commit(bT + 8 * w);
                        if (w == 1 && !key) tc_commit(bE + 8 * (STAGES + s));  // of a row unit V has no other product
                        if (w == 1 && j == n - 1) tc_commit(bXE);
                        return true;
                    };
                    // w = 0: += dS Y1, 1: dV += P Y2 (exact row unit: += P Y1); every 32 columns of dP became 16 of P and 16 of dS
                    auto second_product = [&](int j, int w) {
                        const uint32_t s = (N + j) % STAGES, y = sY + s * C::STAGE_BYTES + (key && w ? C::Y_BYTES : 0);
                        tc_fence_after();
#pragma unroll
                        for (int ks = 0; ks < 8; ++ks)
                            mma_ts(tmem_base + w * D, tmem_base + C::S_COL + 128 + (w ? 0 : 16) + (ks / 2) * 32 + (ks % 2) * 8,
                                   smem_desc_sw128(y + ks * 2048, C::YHALF_BYTES, 1024), idesc2, (j > 0 || ks > 0) ? 1u : 0u);
                        if (key || w == 0) tc_commit(bE + 8 * (w * STAGES + s));
                    };
                    if (n > 0) ok = wait(bX, n_x & 1) && first_product(0, 0) && first_product(0, 1);
                    for (int j = 0; ok && j < n; ++j) {
                        const uint32_t M = N + j;
                        if (!(ok = wait(bP, M & 1))) break;                    // S has been read
                        if (j + 1 < n && !(ok = first_product(j + 1, 0))) break;
                        if (!(ok = wait(bP + 8, M & 1))) break;                // P and dS are there
                        // the first of a unit's second products overwrite the accumulators: those of the unit before have been read
                        if (j == 0 && n_x > 0 && !(ok = wait(bDE, (n_x - 1) & 1))) break;
                        if (key || EXACT) second_product(j, 1);
                        second_product(j, 0);
                        if (j + 1 < n && !(ok = first_product(j + 1, 1))) break;
                    }
                } else {
                    auto first_products = [&](int j) -> bool {
                        const uint32_t M = N + j, s = M % STAGES;
                        if (!wait(bF + 8 * s, (M / STAGES) & 1)) return false;
                        tc_fence_after();
                        const uint32_t y = sY + s * C::STAGE_BYTES;
#pragma unroll
                        for (int w = 0; w < 2; ++w)
#pragma unroll
                            for (int ks = 0; ks < D / 16; ++ks)
                                mma_ss(tmem_base + C::S_COL + C::BUF_COLS * (M % NBUF) + 64 * w,
                                       smem_desc_sw128(sX + w * C::XTILE_BYTES + (ks / 4) * XHALF_BYTES + (ks % 4) * 32, 16, 1024),
                                       smem_desc_sw128(y + w * C::Y_BYTES + (ks / 4) * BLK_BYTES + (ks % 4) * 32, 16, 1024), idesc1, ks > 0);
                        tc_commit(bT + 8 * (M % NBUF));
                        if (j == n - 1) tc_commit(bXE);
                        return true;
                    };
                    if (n > 0) ok = wait(bX, n_x & 1);
                    for (int j = 0; ok && j < min(n, NBUF - 1); ++j) ok = first_products(j);
                    for (int j = 0; ok && j < n; ++j) {
                        // S and dP of block j + NBUF - 1 take the buffers of block j - 1, whose second products were issued before
                        if (j + NBUF - 1 < n && !(ok = first_products(j + NBUF - 1))) break;
                        const uint32_t M = N + j, s = M % STAGES;
                        if (!(ok = wait(bP + 8 * (M % NBUF), (M / NBUF) & 1))) break;
                        // the first of a unit's second products overwrite the accumulators: those of the unit before have been read
                        if (j == 0 && n_x > 0 && !(ok = wait(bDE, (n_x - 1) & 1))) break;
                        tc_fence_after();
                        const uint32_t y = sY + s * C::STAGE_BYTES;
                        // key unit: dK += dS^T Q, dV += P^T dO; row unit: dQ += dS K, and (exact) P K
#pragma unroll
                        for (int w = 0; w < 2; ++w)
                            if (w == 0 || key || EXACT)
#pragma unroll
                                for (int ks = 0; ks < 4; ++ks)
                                    mma_ts(tmem_base + w * D, tmem_base + C::S_COL + C::BUF_COLS * (M % NBUF) + (w ? 0 : 64) + ks * 8,
                                           smem_desc_sw128(y + (key && w ? C::Y_BYTES : 0) + ks * 2048, BLK_BYTES, 1024), idesc2, (j > 0 || ks > 0) ? 1u : 0u);
                        tc_commit(bE + 8 * s);
                    }
                }
                if (!ok) break;
                if (n > 0) {
                    tc_commit(bD);
                    ++n_x;
                }
                N += n;
                mbar_arrive(bUE + 8 * (i & 1));
            }
        }
        __syncwarp();
    } else if (warp < WARPS) {
        reg_inc<ELEMENT_REGS>();
        const int set = warp >> 3, group = 2 * (warp & 3) + ((warp >> 2) & 1), cg = lane & 3;
        const uint32_t lane_addr = tmem_base + ((uint32_t)(16 * group) << 16);
        const float c2 = prm.scale_log2;
        uint32_t N = 0, n_x = 0, n_pair = 0;
        for (uint32_t i = 0;; ++i) {
            if (!__all_sync(0xffffffffu, wait(bUF + 8 * (i & 1), (i >> 1) & 1))) break;
            const Unit& u = ctl->unit[i & 1];
            const int n = u.n;
            if (n < 0) break;
            // a unit's blocks, those of this warp's buffer
            // (A build of its own for exact row units: with a third copy of this code in one the compiler kept the scores in local memory.)
            const bool key = !EXACT && u.key;
            float short_of[2] = {0.f, 0.f};              // exact: the sums of their dS
            auto element_work = [&](auto is_key) {
                constexpr bool KEY = decltype(is_key)::value;
                float nl[2] = {0.f, 0.f}, nd[2] = {0.f, 0.f};
                if (!KEY) {
                    const int row = u.first + 16 * group + (lane >> 2);
                    const long long at = ((long long)u.b * prm.H + u.h) * prm.padded + row;
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        if (row + 8 * e < u.end) {
                            nl[e] = __ldcg(prm.nlse + at + 8 * e);
                            nd[e] = __ldcg(prm.ndelta + at + 8 * e);
                        }
                }
                Walk at(u);
                const int per_head = u.per_head, free_from = u.free[2 * group + set].x;
                const uint32_t free_count = u.free[2 * group + set].y;
                // Scores of columns that the thread's two rows do not see become -inf: numbers 4 k + 2 e, + 1 of half x are columns 32 x + 8 k + 2 cg, + 1 of
                // row e.
                auto hide = [&](int col0, auto&& score) {
                    const int row = u.first + 16 * group + (lane >> 2), off = u.keys - u.rows, end = u.end;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int r = row + 8 * e;
                        uint32_t bits[2];
                        if (KEY) {
                            int lo, hi, full_lo, full_hi;
                            rows_of_key(prm.w, r, u.rows, off, lo, hi);
                            full_rows(prm.w, u.rows, off, full_lo, full_hi);
#pragma unroll
                            for (int x = 0; x < 2; ++x) {
                                const int c0 = col0 + 32 * x;
                                bits[x] = (bits_below(hi - c0) & ~bits_below(lo - c0)) | (bits_below(full_hi - c0) & ~bits_below(full_lo - c0));
                            }
                        } else {
                            prm.w.seen_bits(r + off, r < end ? u.keys : 0, col0, bits);
                        }
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            const uint32_t w = bits[x] >> (2 * cg);
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                if (!(w >> (8 * k) & 1u)) score(x, 4 * k + 2 * e) = 0xff800000u;
                                if (!(w >> (8 * k + 1) & 1u)) score(x, 4 * k + 2 * e + 1) = 0xff800000u;
                            }
                        }
                    }
                };
                // dS of a column whose row sees one key is 0 (where every row of a block sees all of the warp's keys, two at least, there is none)
                auto mark = [&](auto looked_at, uint64_t cd, float2& g) {
                    if (KEY && decltype(looked_at)::value) {
                        const float2 d = of_pair(cd);
                        if (d.x == INFINITY) g.x = 0.f;
                        if (d.y == INFINITY) g.y = 0.f;
                    }
                };
                if constexpr (WIDE) {
                    for (int j = 0; j < n; ++j, at.next(per_head)) {
                        const uint32_t M = N + j, buf = M % STAGES;
                        int col0 = 0;
                        bool act = true, compare = false;
                        if ((uint32_t)(at.j - free_from) >= free_count) {
                            col0 = WIDTH * u.blocks.at(at.j) + 64 * set;
                            const int4 whole = u.whole[group];
                            const int3 reach = u.reach[group];
                            act = (col0 < reach.y && col0 + 64 > reach.x) || col0 < reach.z;
                            compare = !((col0 >= whole.x && col0 + 64 <= whole.y) || (col0 >= whole.z && col0 + 64 <= whole.w));
                        }
                        const uint32_t tS = lane_addr + C::S_COL + 64 * set, tP = tS + 128;
                        const uint64_t* const st = reinterpret_cast<const uint64_t*>(stats + buf * C::STAT_BYTES + 256 * set) + cg;
                        uint32_t s[32];
                        // (nothing up to the end of the unit depends on a wait's result; the flag is looked at once in a while)
                        if (j % ABORT_EVERY == 0 && __any_sync(0xffffffffu, ctl->abort_flag)) return;
                        if (KEY) wait(bF + 8 * buf, (M / STAGES) & 1);             // nlse and ndelta, read below
                        wait(bT, M & 1);
                        __syncwarp();
                        tc_fence_after();
                        if (act) {
                            tmem_ld16x256_x8(tS, s);
                            tc_wait_ld();
                        }
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(bP);
                        if (act) {
                            if (compare) hide(col0, [&](int x, int i) -> uint32_t& { return s[16 * x + i]; });
#pragma unroll
                            for (int k = 0; k < 8; ++k) {
                                uint64_t cl;
                                if (KEY) cl = st[4 * k];
#pragma unroll
                                for (int e = 0; e < 2; ++e) {
                                    const uint64_t sv = pair_of(__uint_as_float(s[4 * k + 2 * e]), __uint_as_float(s[4 * k + 2 * e + 1]));
                                    const float2 p = of_pair(fma2(sv, pair_of(c2, c2), KEY ? cl : pair_of(nl[e], nl[e])));
                                    s[4 * k + 2 * e] = __float_as_uint(ex2(p.x));
                                    s[4 * k + 2 * e + 1] = __float_as_uint(ex2(p.y));
                                }
                            }
                        }
                        wait(bT + 8, M & 1);
                        __syncwarp();
                        tc_fence_after();
                        auto second_step = [&](auto looked_at) {
#pragma unroll
                            for (int x = 0; x < 2; ++x) {
                                uint32_t pp[8], pd[8], d[16];
                                tmem_ld16x256_x4(tP + 32 * x, d);
                                tc_wait_ld();
                                if (EXACT) {             // (before dS, for registers)
#pragma unroll
                                    for (int i = 0; i < 8; ++i) pp[i] = pack16<TYPE>(__uint_as_float(s[16 * x + 2 * i]), __uint_as_float(s[16 * x + 2 * i + 1]));
                                    tmem_st16x128_x4(tP + 32 * x, pp);
                                }
#pragma unroll
                                for (int k = 0; k < 4; ++k) {
                                    uint64_t cd;
                                    if (KEY) cd = st[WIDTH / 2 + 4 * (4 * x + k)];
#pragma unroll
                                    for (int e = 0; e < 2; ++e) {
                                        const int i = 16 * x + 4 * k + 2 * e;
                                        const uint64_t dv = pair_of(__uint_as_float(d[4 * k + 2 * e]), __uint_as_float(d[4 * k + 2 * e + 1]));
                                        const uint64_t p = pair_of(__uint_as_float(s[i]), __uint_as_float(s[i + 1]));
                                        float2 g = of_pair(mul2(p, fma2(dv, pair_of(1.f, 1.f), KEY ? cd : pair_of(nd[e], nd[e]))));
                                        mark(looked_at, cd, g);
                                        if (EXACT) short_of[e] += g.x + g.y;
                                        if (KEY) pp[2 * k + e] = pack16<TYPE>(__uint_as_float(s[i]), __uint_as_float(s[i + 1]));
                                        pd[2 * k + e] = pack16<TYPE>(g.x, g.y);
                                    }
                                }
                                if (KEY) tmem_st16x128_x4(tP + 32 * x, pp);
                                tmem_st16x128_x4(tP + 32 * x + 16, pd);
                            }
                        };
                        if (!act) {
                            uint32_t zero[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
#pragma unroll
                            for (int x = 0; x < 4; ++x) tmem_st16x128_x4(tP + 16 * x, zero);
                        } else if (KEY && compare) {
                            second_step(std::true_type());
                        } else {
                            second_step(std::false_type());
                        }
                        tc_wait_st();
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(bP + 8);
                    }
                } else {
                    for (int j = 0; j < n; ++j, at.next(per_head)) {
                        const uint32_t M = N + j;
                        if ((int)(M & 1) != set) continue;
                        int col0 = 0;
                        bool act = true, compare = false;
                        if ((uint32_t)(at.j - free_from) >= free_count) {
                            col0 = 64 * u.blocks.at(at.j);
                            const int4 whole = u.whole[group];
                            const int3 reach = u.reach[group];
                            act = (col0 < reach.y && col0 + 64 > reach.x) || col0 < reach.z;
                            compare = !((col0 >= whole.x && col0 + 64 <= whole.y) || (col0 >= whole.z && col0 + 64 <= whole.w));
                        }
                        const uint32_t buf = M % NBUF, tS = lane_addr + C::S_COL + C::BUF_COLS * buf, tP = tS + 64;
                        if (j % ABORT_EVERY < 2 && __any_sync(0xffffffffu, ctl->abort_flag)) return;
                        if (KEY) wait(bF + 8 * (M % STAGES), (M / STAGES) & 1);    // nlse and ndelta of the block, read below
                        wait(bT + 8 * buf, (M / NBUF) & 1);
                        __syncwarp();
                        tc_fence_after();
                        if (act) {
                            uint32_t s[2][16], d[2][16];
#pragma unroll
                            for (int x = 0; x < 2; ++x) {
                                tmem_ld16x256_x4(tS + 32 * x, s[x]);
                                tmem_ld16x256_x4(tP + 32 * x, d[x]);
                            }
                            tc_wait_ld();
                            if (compare) {
                                hide(col0, [&](int x, int i) -> uint32_t& { return s[x][i]; });
                            }
                            const uint64_t* const st = reinterpret_cast<const uint64_t*>(stats + (M % STAGES) * C::STAT_BYTES) + cg;
                            auto both_steps = [&](auto looked_at) {
#pragma unroll
                                for (int x = 0; x < 2; ++x) {
                                    uint32_t pp[8], pd[8];
#pragma unroll
                                    for (int k = 0; k < 4; ++k) {
                                        uint64_t cl, cd;
                                        if (KEY) {
                                            cl = st[4 * (4 * x + k)];
                                            cd = st[32 + 4 * (4 * x + k)];
                                        }
#pragma unroll
                                        for (int e = 0; e < 2; ++e) {
                                            const uint64_t sv = pair_of(__uint_as_float(s[x][4 * k + 2 * e]), __uint_as_float(s[x][4 * k + 2 * e + 1]));
                                            const uint64_t dv = pair_of(__uint_as_float(d[x][4 * k + 2 * e]), __uint_as_float(d[x][4 * k + 2 * e + 1]));
                                            float2 p = of_pair(fma2(sv, pair_of(c2, c2), KEY ? cl : pair_of(nl[e], nl[e])));
                                            p.x = ex2(p.x);
                                            p.y = ex2(p.y);
                                            if (KEY || EXACT) pp[2 * k + e] = pack16<TYPE>(p.x, p.y);
                                            float2 g = of_pair(mul2(pair_of(p.x, p.y), fma2(dv, pair_of(1.f, 1.f), KEY ? cd : pair_of(nd[e], nd[e]))));
                                            mark(looked_at, cd, g);
                                            if (EXACT) short_of[e] += g.x + g.y;
                                            pd[2 * k + e] = pack16<TYPE>(g.x, g.y);
                                        }
                                    }
                                    // over what this warp has read: the first half's numbers lie in the first quarter of the buffer
                                    if (KEY || EXACT) tmem_st16x128_x4(tS + 16 * x, pp);
                                    tmem_st16x128_x4(tP + 16 * x, pd);
                                }
                            };
                            if (KEY && compare) both_steps(std::true_type());
                            else both_steps(std::false_type());
                        } else {
                            uint32_t zero[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
#pragma unroll
                            for (int x = 0; x < 2; ++x) {
                                if (KEY || EXACT) tmem_st16x128_x4(tS + 16 * x, zero);
                                tmem_st16x128_x4(tP + 16 * x, zero);
                            }
                        }
                        tc_wait_st();
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(bP + 8 * buf);
                    }
                }
            };
            if constexpr (EXACT) {
                element_work(std::false_type());
            } else {
                if (key) element_work(std::true_type());
                else element_work(std::false_type());
            }
            float nd[2] = {0.f, 0.f};                    // of a row unit, minus delta of the thread's two rows, again
            if (!key) {
                const int row = u.first + 16 * group + (lane >> 2);
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    if (row + 8 * e < u.end) nd[e] = __ldcg(prm.ndelta + ((long long)u.b * prm.H + u.h) * prm.padded + row + 8 * e);
            }
            // e of the thread's two rows: of its lane quad's columns, then of both sets
            float e_row[2] = {0.f, 0.f};
            if constexpr (EXACT) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float x = short_of[e];
                    x += __shfl_xor_sync(0xffffffffu, x, 1);
                    x += __shfl_xor_sync(0xffffffffu, x, 2);
                    if (cg == 0) ctl->short_of[i & 1][warp][(lane >> 2) + 8 * e] = x;
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(bPair + 8 * group);
                wait(bPair + 8 * group, n_pair++ & 1);
                __syncwarp();
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int r = (lane >> 2) + 8 * e, low = warp & 7;
                    e_row[e] = ctl->short_of[i & 1][low][r] + ctl->short_of[i & 1][low + 8][r];
                    const int row = u.first + 16 * group + r;
                    // (of a row that sees one key e is not a number, and its mark stays)
                    if (set == 0 && cg == 0 && row < u.end && nd[e] != INFINITY)
                        __stcg(prm.ndelta + ((long long)u.b * prm.H + u.h) * prm.padded + row, nd[e] - e_row[e]);
                }
            }
            // the results: of a key unit half of the warps dK, half dV; of a row unit half of dQ's channels each
            if (n > 0) wait(bD, n_x & 1);
            if (!__all_sync(0xffffffffu, !ctl->abort_flag)) break;
            tc_fence_after();
            const int row = u.first + 16 * group + (lane >> 2);
            const bool r0 = row < u.end, r1 = row + 8 < u.end;
            const int chunks = key ? D / 32 : D / 64, ch0 = key ? 0 : set * chunks, col = key ? set * D : 0;
            const Rows& to = key ? (set ? prm.dv : prm.dk) : prm.dq;
            const float f = key && set ? 1.f : prm.scale;
            char* const o_lo = to.row(u.b, u.h, row) + 16 * cg;
            char* const o_hi = o_lo + 16 * to.n;
            float* const part = u.slot >= 0 ? prm.partial + ((long long)u.slot * 128 + 16 * group + (lane >> 2)) * (2 * D) + col : nullptr;
            for (int ch = ch0; ch < ch0 + chunks; ++ch) {
                uint32_t o[16];
                if (n > 0) {
                    tmem_ld16x256_x4(lane_addr + col + ch * 32, o);
                    tc_wait_ld();
                } else {
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[e] = 0u;
                }
                if (part) {                              // of a shared-out tile: 32 bits, not scaled
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        __stcg(reinterpret_cast<float2*>(part + 32 * ch + 8 * k + 2 * cg), make_float2(__uint_as_float(o[4 * k]), __uint_as_float(o[4 * k + 1])));
                        __stcg(reinterpret_cast<float2*>(part + 8 * 2 * D + 32 * ch + 8 * k + 2 * cg),
                               make_float2(__uint_as_float(o[4 * k + 2]), __uint_as_float(o[4 * k + 3])));
                    }
                    continue;
                }
                if constexpr (EXACT) {
                    uint32_t pk[16];
                    if (n > 0) {
                        tmem_ld16x256_x4(lane_addr + D + ch * 32, pk);
                        tc_wait_ld();
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(fmaf(-e_row[e >> 1 & 1], __uint_as_float(pk[e]), __uint_as_float(o[e])));
                    }
                }
                if (!key) {                              // rows that see one key
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (nd[e >> 1 & 1] == INFINITY) o[e] = 0u;
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
                __syncwarp();
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (n > 0) mbar_arrive(bDE);
                mbar_arrive(bUE + 8 * (i & 1));
            }
            if (n > 0) ++n_x;
            N += n;
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

// The results of shared-out key tiles, added up in the order of their parts: a thread eight channels of a key's dK or dV.
template <int D, int TYPE>
__global__ void __launch_bounds__(256) add_parts_kernel(const __grid_constant__ Params p, int B, int tiles) {
    grid_dependency_wait();
    grid_dependency_launch();
    constexpr int PER_ROW = 2 * D / 8;
    const int x = blockIdx.x * 256 + threadIdx.x, c = x % PER_ROW, row = x / PER_ROW % 128, t = x / PER_ROW / 128;
    if (t >= tiles) return;
    const int heads = B * p.H_kv, tile = t / heads, at = t - tile * heads, b = at / p.H_kv, h = at - b * p.H_kv, key = 128 * tile + row;
    if (key >= p.w.keys(b)) return;
    float sum[8] = {};
    for (int i = 0; i < p.parts; ++i) {
        const float4* from = reinterpret_cast<const float4*>(p.partial + (((long long)t * p.parts + i) * 128 + row) * (2 * D) + 8 * c);
        const float4 a = __ldcg(from), bb = __ldcg(from + 1);
        sum[0] += a.x; sum[1] += a.y; sum[2] += a.z; sum[3] += a.w;
        sum[4] += bb.x; sum[5] += bb.y; sum[6] += bb.z; sum[7] += bb.w;
    }
    const bool value = 8 * c >= D;
    const float f = value ? 1.f : p.scale;
    char* to = (value ? p.dv : p.dk).row(b, h, key) + 2 * (8 * c - (value ? D : 0));
    *reinterpret_cast<uint4*>(to) = make_uint4(pack16<TYPE>(sum[0] * f, sum[1] * f), pack16<TYPE>(sum[2] * f, sum[3] * f),
                                               pack16<TYPE>(sum[4] * f, sum[5] * f), pack16<TYPE>(sum[6] * f, sum[7] * f));
}

// Minus log sum exp in base 2 and minus delta of every query row, padded to whole blocks with rows that have no P.  Bound by HBM: O and dO once.
template <int D, int TYPE>
__global__ void __launch_bounds__(256) row_stats_kernel(const Rule w, const Rows out, const Rows dout, const float* lse, float* nlse, float* ndelta,
                                                        int H, int padded) {
    constexpr int LPR = D / 8;                           // lanes of a row, 16 bytes each
    constexpr int AT_ONCE = 4, PER = 256 / LPR;          // rows of a lane, rows of a pass
    const int lane = threadIdx.x % LPR, i0 = blockIdx.x * (PER * AT_ONCE) + threadIdx.x / LPR, h = blockIdx.y % H, b = blockIdx.y / H;
    grid_dependency_wait();
    const int rows = w.rows(b), keys = w.keys(b);
    uint4 o[AT_ONCE], d[AT_ONCE];
    float l[AT_ONCE];
#pragma unroll
    for (int x = 0; x < AT_ONCE; ++x) {
        const int i = i0 + x * PER;
        o[x] = d[x] = make_uint4(0, 0, 0, 0);
        l[x] = -INFINITY;
        if (i < rows) {
            o[x] = __ldcg(reinterpret_cast<const uint4*>(out.row(b, h, i) + 16 * lane));
            d[x] = __ldcg(reinterpret_cast<const uint4*>(dout.row(b, h, i) + 16 * lane));
            if (lane == 0) l[x] = __ldcg(lse + ((long long)b * H + h) * w.n_q + i);
        }
    }
    grid_dependency_launch();
#pragma unroll
    for (int x = 0; x < AT_ONCE; ++x) {
        const int i = i0 + x * PER;
        const uint32_t ow[4] = {o[x].x, o[x].y, o[x].z, o[x].w}, dw[4] = {d[x].x, d[x].y, d[x].z, d[x].w};
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 a = unpack16<TYPE>(ow[e]), c = unpack16<TYPE>(dw[e]);
            sum = fmaf(a.x, c.x, fmaf(a.y, c.y, sum));
        }
#pragma unroll
        for (int z = 1; z < LPR; z <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, z);
        if (lane == 0 && i < padded) {
            const long long at = ((long long)b * H + h) * padded + i;
            nlse[at] = l[x] == -INFINITY ? -INFINITY : l[x] * -1.4426950408889634f;
            ndelta[at] = i < rows && w.count(i + keys - rows, keys) == 1 ? INFINITY : -sum;
        }
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
    for (const void* kernel : {(const void*)window_back_kernel<D, TYPE, false>, (const void*)window_back_kernel<D, TYPE, true>}) {
        if ((e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes<D>())) != cudaSuccess) return e;
        // the warps that take registers wait for them: a build that is launched with fewer would wait for good
        cudaFuncAttributes attr;
        if ((e = cudaFuncGetAttributes(&attr, kernel)) != cudaSuccess) return e;
        if (attr.numRegs * NTHREADS < 32 * (WARPS * ELEMENT_REGS + 4 * LIGHT_REGS)) return cudaErrorInvalidKernelImage;
    }
    done.fetch_or(bit, std::memory_order_release);
    return cudaSuccess;
}

int padded_rows(const rapid3_window* w) { return (w->n_q + 127) / 128 * 128; }
int64_t stat_floats(const rapid3_window* w) { return (int64_t)w->B * w->H * padded_rows(w); }

// Tiles of first tokens, and how many units share one: so many that none takes longer than half of what an SM has to do in the mean, all
// sequences taken as full.
void sharing(const rapid3_window* w, int& sink_tiles, int& parts) {
    sink_tiles = 0;
    parts = 1;
    if (w->left < 0 || w->n_sink == 0) return;
    const long long tiles = (w->n_kv + 127) / 128, row_tiles = (w->n_q + 127) / 128, row_blocks = (w->n_q + 63) / 64, key_blocks = (w->n_kv + 63) / 64;
    sink_tiles = (int)std::min<long long>(tiles, (std::min(w->n_sink, w->n_kv) + 127) / 128);
    const long long near = (long long)w->left + (w->right < 0 ? std::max(w->n_q, w->n_kv) : w->right) + 192, group = w->H / w->H_kv;
    const long long sink = group * row_blocks, other = group * std::min(row_blocks, near / 64);
    const long long total = (long long)w->B * w->H_kv * (sink_tiles * sink + (tiles - sink_tiles) * other) +
                            (long long)w->B * w->H * row_tiles * std::min(key_blocks, near / 64 + (w->n_sink + 63) / 64);
    const long long most = std::max<long long>(48, total / SM_COUNT / 2), slots = (long long)sink_tiles * w->B * w->H_kv;
    parts = (int)std::min<long long>(std::min<long long>(MAX_PARTS, (sink + most - 1) / most), std::max<long long>(1, MAX_SLOTS / slots));
}

// The first row tiles that are looked at for rows which see fewer than EXACT_FROM keys, by their first and last rows: none, some at the beginning, or (where
// that is not for the host to say) all.  every: each tile surely holds such rows.
// Where the first tile's rows are full, or a tile's first ones, rows behind them that see 129 keys and more may go without (fewer they never see there: their
// window is 256 wide, or the last tile's rows see few too): their dq is off by 0.61 to 0.62 half steps in the mean square, for 0.60 to 0.61 with the exact pass.
int few_tiles(const rapid3_window* w, bool& every) {
    const int tiles = (w->n_q + 127) / 128;
    every = false;
    if (w->q_len || w->kv_len || w->n_q > w->n_kv) return tiles;
    Rule rule = rule_of(w);
    auto few = [&](int tile) {
        const int off = w->n_kv - w->n_q, first = 128 * tile + off, last = std::min(128 * tile + 127, w->n_q - 1) + off;
        return std::min(rule.count(first, w->n_kv), rule.count(last, w->n_kv)) < EXACT_FROM;
    };
    int n = 0;
    if (w->left >= 0 && w->right >= 0 && (long long)w->left + w->right + 1 + w->n_sink < EXACT_FROM && w->n_full == 0) n = tiles;
    while (n < tiles && few(n)) ++n;
    every = n == tiles;
    // the rows behind see a whole window or the keys of all that are in front, but for those at the end
    return n < tiles && few(tiles - 1) ? tiles : n;
}

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
    float* const ndelta = stats + stat_floats(w);
    p.nlse = stats;
    p.ndelta = ndelta;
    p.partial = ndelta + stat_floats(w);
    p.H = w->H;
    p.H_kv = w->H_kv;
    p.group = w->H / w->H_kv;
    p.scale = w->softmax_scale;
    p.scale_log2 = w->softmax_scale * 1.4426950408889634f;
    p.dq = rows_arg(dq);
    p.dk = rows_arg(dk);
    p.dv = rows_arg(dv);
    p.key_tiles = (w->n_kv + 127) / 128;
    p.row_tiles = (w->n_q + 127) / 128;
    sharing(w, p.sink_tiles, p.parts);
    const long long full = std::min<long long>(w->n_q, w->n_full ? (long long)w->n_full + w->n_q - w->n_kv : 0);    // rows, of full sequences
    p.full_tiles = full > 0 ? (int)((full + 127) / 128) : 0;
    p.last_first = w->left < 0 && w->right >= 0;
    const int key_heads = w->B * w->H_kv, heads = w->B * w->H;
    p.sink_units = key_heads * p.sink_tiles * p.parts;
    p.key_units = p.sink_units + key_heads * (p.key_tiles - p.sink_tiles);
    p.full_units = p.key_units + heads * p.full_tiles;
    const int units = p.full_units + heads * (p.row_tiles - p.full_tiles);
    constexpr int PER = 4 * 256 / (D / 8);
    if (launch_kernel(row_stats_kernel<D, TYPE>, dim3((p.padded + PER - 1) / PER, heads), dim3(256), 0, s, p.w, rows_arg(out), rows_arg(dout), lse,
                      stats, ndelta, w->H, p.padded) != cudaSuccess)
        return RAPID3_ERR_CUDA;
    bool every;
    p.few_tiles = few_tiles(w, every);
    p.pass = p.few_tiles > 0 ? 1 : 0;
    if (p.pass == 1) {
        if (launch_kernel(window_back_kernel<D, TYPE, true>, dim3(heads * p.few_tiles), dim3(NTHREADS), smem_bytes<D>(), s, tq, tk, tv, td, p, w->B) != cudaSuccess)
            return RAPID3_ERR_CUDA;
        p.pass = 2;
    }
    if (launch_kernel(window_back_kernel<D, TYPE, false>, dim3(every ? p.key_units : units), dim3(NTHREADS), smem_bytes<D>(), s, tq, tk, tv, td, p, w->B) != cudaSuccess)
        return RAPID3_ERR_CUDA;
    const int shared = key_heads * p.sink_tiles;
    if (p.parts > 1 && launch_kernel(add_parts_kernel<D, TYPE>, dim3((shared * 128 * (2 * D / 8) + 255) / 256), dim3(256), 0, s, p, w->B, shared) != cudaSuccess)
        return RAPID3_ERR_CUDA;
    return RAPID3_OK;
}

}  // namespace

cudaError_t window_back_status(int* value, bool clear) {
    const int zero = 0;
    return clear ? cudaMemcpyToSymbol(status_word, &zero, sizeof(int)) : cudaMemcpyFromSymbol(value, status_word, sizeof(int));
}

extern "C" {

int64_t rapid3_window_workspace_bytes(const rapid3_window* w) {
    const int r = window::check(w);
    if (r) return r;
    int sink_tiles, parts;
    sharing(w, sink_tiles, parts);
    const int64_t slots = parts > 1 ? (int64_t)w->B * w->H_kv * sink_tiles * parts : 0;
    return (2 * stat_floats(w) + slots * 128 * 2 * w->D) * sizeof(float);
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
