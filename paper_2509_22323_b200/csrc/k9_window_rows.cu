// K9: attention with a window and first tokens for few query rows, from a cache: the single tokens of serving.  The rows of all query
// heads that share a key head (16 at most) are one side of mma.m16n8k16, so K and V are read once; tcgen05's tiles of 128 rows would stand
// empty.  Bound by HBM: 4 D bytes a visible key.  Up to eight rows (NARROW) are the products' columns, K and V^T the first operands:
// S^T = K Q^T, O^T = V^T P^T, where half of a sixteen-row tile would be empty and its accumulators take the registers of loads on their way.
//
// A warp takes sixteen keys at a time straight into the registers that the products want them in, without shared memory: the
// channels of a product's contraction may come in any order that Q and K share, and the columns of the second one are channels
// in any order, so both fragments are made of 16-byte loads: K by key (four lanes 64 bytes of one), V by key (eight lanes 128 bytes),
// pairs of keys put together with byte permutes.  The next sixteen keys' loads go out as soon as the registers are free, so that nearly all of
// a warp's 8 KB (D = 128) are always on their way.
//
// The keys of a (sequence, key head) are split over the warps of a cluster of thread blocks.  Their partial results (sums not divided, row
// sums and maxima) meet in shared memory, the thread blocks' in distributed shared memory, each doing a share of the channels: one
// launch, no workspace, and an order that is always the same.
// Measured: 64 sequences of 5461 to 16384 tokens, 64 heads on 8, D = 128, 4100 keys each: 1.07 GB in 187 us, 5.7 TB/s, 0.87 of a copy's rate.
#include <float.h>

#include <algorithm>
#include <atomic>

#include "window.cuh"

using namespace window;

namespace {

constexpr int WARPS = 4, CHUNK = 16, MAX_ROWS = 16, MAX_CLUSTER = 16;

struct RowsParams {
    Rule w;
    Rows q, k, v, out;
    float* lse;
    int H, H_kv, group;          // query heads of a key head
    float scale_log2;
};

template <int TYPE>
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (TYPE == RAPID3_BF16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// (past the L1: what is read may have been written by the kernel right in front)
__device__ __forceinline__ uint4 load16(const char* p) { return __ldcg(reinterpret_cast<const uint4*>(p)); }
__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ uint32_t cluster_size() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
}
__device__ __forceinline__ float peer_float(uint32_t addr, uint32_t rank) {
    float v;
    asm volatile("{\n\t.reg .u32 a;\n\tmapa.shared::cluster.u32 a, %1, %2;\n\tld.shared::cluster.f32 %0, [a];\n\t}" : "=f"(v) : "r"(addr), "r"(rank) : "memory");
    return v;
}

template <int TYPE, int D, bool NARROW>
__global__ void __launch_bounds__(32 * WARPS, NARROW ? (D == 128 ? 3 : 4) : 2) window_rows_kernel(const __grid_constant__ RowsParams p) {
    constexpr int KV = D / 32;                           // 16-byte loads of a lane for eight keys of K, or for two keys of V by halves: D / 64 blocks
    constexpr int DB = D / 64;
    constexpr int ROWS = NARROW ? 8 : MAX_ROWS;
    __shared__ float o_sh[WARPS][ROWS][D + 4];
    __shared__ float m_sh[WARPS][ROWS], l_sh[WARPS][ROWS];
    __shared__ float weight[WARPS][ROWS];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane >> 2, c = lane & 3;
    const int rank = (int)cluster_rank(), size = (int)cluster_size();
    const int pair = blockIdx.x / size, b = pair / p.H_kv, hk = pair - b * p.H_kv;
    const int n_rows = p.group * p.w.n_q;
    grid_dependency_wait();
    const int rows = p.w.rows(b), keys = p.w.keys(b);

    // Row r is query r % n_q of head r / n_q of the group.  The thread's scores are those of rows g and g + 8, or (NARROW) 2 c and 2 c + 1.
    int lo[2], hi[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const int r = NARROW ? 2 * c + x : g + 8 * x, i = r - r / p.w.n_q * p.w.n_q;
        lo[x] = hi[x] = 0;
        if (r < n_rows && i < rows) p.w.seen(i + keys - rows, keys, lo[x], hi[x]);
    }
    // Q as the products want it: of rows g and g + 8, or g alone; channels in the order of 16-byte loads, which K's are in too
    uint32_t qf[D / 16][NARROW ? 2 : 4];
#pragma unroll
    for (int x = 0; x < (NARROW ? 1 : 2); ++x) {
        const int r = g + 8 * x, head = r / p.w.n_q, i = r - head * p.w.n_q;
        const bool there = r < n_rows && i < rows;
        const char* src = p.q.row(b, hk * p.group + (there ? head : 0), there ? i : 0) + 16 * c;
#pragma unroll
        for (int s = 0; s < KV; ++s) {
            const uint4 v = there ? load16(src + 64 * s) : make_uint4(0, 0, 0, 0);
            if constexpr (NARROW) {
                qf[2 * s][0] = v.x; qf[2 * s][1] = v.y;
                qf[2 * s + 1][0] = v.z; qf[2 * s + 1][1] = v.w;
            } else {
                qf[2 * s][x] = v.x; qf[2 * s][2 + x] = v.y;
                qf[2 * s + 1][x] = v.z; qf[2 * s + 1][2 + x] = v.w;
            }
        }
    }
    // the keys that any row sees: first ones, then a window
    const bool any0 = hi[0] > 0, any1 = hi[1] > 0;
    int from = min(any0 ? lo[0] : keys, any1 ? lo[1] : keys), to = max(hi[0], hi[1]);
    from = __reduce_min_sync(0xffffffffu, from);
    to = __reduce_max_sync(0xffffffffu, to);
    from = min(from, to);
    const int first_end = min(min(p.w.n_sink, from), to);
    const int first_chunks = (first_end + CHUNK - 1) / CHUNK, chunks = first_chunks + (to - from + CHUNK - 1) / CHUNK;

    const char* kp = p.k.row(b, hk, 0) + 16 * c;
    const char* vp = p.v.row(b, hk, 0) + 16 * g;
    const long long kn = 2 * p.k.n, vn = 2 * p.v.n;
    uint4 kr[2][KV], vr[4][DB];
    auto span = [&](int chunk, int& base, int& end) {
        const bool f = chunk < first_chunks;
        base = f ? chunk * CHUNK : from + (chunk - first_chunks) * CHUNK;
        end = f ? first_end : to;
    };
    auto load_k = [&](int chunk) {
        int base, end;
        span(chunk, base, end);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int key = base + 8 * t + g;
#pragma unroll
            for (int s = 0; s < KV; ++s) kr[t][s] = key < end ? load16(kp + key * kn + 64 * s) : make_uint4(0, 0, 0, 0);
        }
    };
    auto load_v = [&](int chunk) {
        int base, end;
        span(chunk, base, end);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int key = base + 2 * c + (t & 1) + 8 * (t >> 1);
#pragma unroll
            for (int s = 0; s < DB; ++s) vr[t][s] = key < end ? load16(vp + key * vn + 128 * s) : make_uint4(0, 0, 0, 0);
        }
    };
    constexpr int TILES = NARROW ? D / 16 : D / 8;       // products for O: sixteen channels of eight rows each, or eight of sixteen
    float o[TILES][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
    for (int t = 0; t < TILES; ++t) o[t][0] = o[t][1] = o[t][2] = o[t][3] = 0.f;
    // a thread block's chunks lie side by side, its warps take them by turns
    const int last = (int)((long long)chunks * (rank + 1) / size);
    int chunk = (int)((long long)chunks * rank / size) + warp;
    if (chunk < last) {
        load_k(chunk);
        load_v(chunk);
    }
    for (; chunk < last; chunk += WARPS) {
        // sixteen keys' scores, of the thread's row x and key base + key_of(x, y) at s[x][y]
        float s[2][4];
        if constexpr (NARROW) {
            float a[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int x = 0; x < KV; ++x) {
                const uint32_t k0[4] = {kr[0][x].x, kr[1][x].x, kr[0][x].y, kr[1][x].y}, k1[4] = {kr[0][x].z, kr[1][x].z, kr[0][x].w, kr[1][x].w};
                mma16816<TYPE>(a, k0, qf[2 * x][0], qf[2 * x][1]);
                mma16816<TYPE>(a, k1, qf[2 * x + 1][0], qf[2 * x + 1][1]);
            }
            s[0][0] = a[0]; s[1][0] = a[1]; s[0][1] = a[2]; s[1][1] = a[3];
        } else {
            float a[2][4];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                a[t][0] = a[t][1] = a[t][2] = a[t][3] = 0.f;
#pragma unroll
                for (int x = 0; x < KV; ++x) {
                    const uint32_t q0[4] = {qf[2 * x][0], qf[2 * x][1], qf[2 * x][NARROW ? 0 : 2], qf[2 * x][NARROW ? 0 : 3]};
                    const uint32_t q1[4] = {qf[2 * x + 1][0], qf[2 * x + 1][1], qf[2 * x + 1][NARROW ? 0 : 2], qf[2 * x + 1][NARROW ? 0 : 3]};
                    mma16816<TYPE>(a[t], q0, kr[t][x].x, kr[t][x].y);
                    mma16816<TYPE>(a[t], q1, kr[t][x].z, kr[t][x].w);
                }
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int y = 0; y < 2; ++y) s[x][2 * t + y] = a[t][2 * x + y];
            }
        }
        const bool more = chunk + WARPS < last;
        if (more) load_k(chunk + WARPS);
        int base, end;
        span(chunk, base, end);
        constexpr int PER = NARROW ? 2 : 4;              // scores of a row
        float top[2] = {-INFINITY, -INFINITY}, shift[2], f[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
#pragma unroll
            for (int y = 0; y < PER; ++y) {
                const int j = base + (NARROW ? g + 8 * y : 8 * (y >> 1) + 2 * c + (y & 1));
                const bool seen = j < min(hi[x], end) && (j >= lo[x] || j < p.w.n_sink);
                s[x][y] = seen ? s[x][y] * p.scale_log2 : -INFINITY;
                top[x] = fmaxf(top[x], s[x][y]);
            }
#pragma unroll
            for (int z = NARROW ? 4 : 1; z < (NARROW ? 32 : 4); z <<= 1) top[x] = fmaxf(top[x], __shfl_xor_sync(0xffffffffu, top[x], z));
            const float next = fmaxf(m[x], top[x]);
            shift[x] = next == -INFINITY ? 0.f : next;
            f[x] = ptx::ex2(m[x] - shift[x]);            // 0 where nothing was seen so far
            l[x] *= f[x];
            m[x] = next;
#pragma unroll
            for (int y = 0; y < PER; ++y) {
                s[x][y] = ptx::ex2(s[x][y] - shift[x]);
                l[x] += s[x][y];
            }
        }
        if (__any_sync(0xffffffffu, f[0] != 1.f || f[1] != 1.f))
#pragma unroll
            for (int t = 0; t < TILES; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[t][e] *= f[NARROW ? e & 1 : e >> 1];
        uint32_t w[4][DB][4];                            // V: of four keys, two channels a word
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                w[t][db][0] = vr[t][db].x; w[t][db][1] = vr[t][db].y; w[t][db][2] = vr[t][db].z; w[t][db][3] = vr[t][db].w;
            }
        if constexpr (NARROW) {
            // P^T with its keys along the products' contraction: two 8 x 8 transposes
            uint32_t p0 = pack16<TYPE>(s[0][0], s[1][0]), p1 = pack16<TYPE>(s[0][1], s[1][1]);
            asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %0;" : "+r"(p0));
            asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %0;" : "+r"(p1));
#pragma unroll
            for (int t = 0; t < TILES; ++t) {            // rows g, g + 8 of product t are channels 8 g + t and 64 more (D = 64: 8 g + t and 4 more)
                const int second = D == 128 ? t : t + 4, db = D == 128 ? 1 : 0;
                const uint32_t pick0 = t & 1 ? 0x7632u : 0x5410u, pick1 = second & 1 ? 0x7632u : 0x5410u;
                const uint32_t a[4] = {__byte_perm(w[0][0][t >> 1], w[1][0][t >> 1], pick0), __byte_perm(w[0][db][second >> 1], w[1][db][second >> 1], pick1),
                                       __byte_perm(w[2][0][t >> 1], w[3][0][t >> 1], pick0), __byte_perm(w[2][db][second >> 1], w[3][db][second >> 1], pick1)};
                mma16816<TYPE>(o[t], a, p0, p1);
            }
        } else {
            const uint32_t pf[4] = {pack16<TYPE>(s[0][0], s[0][1]), pack16<TYPE>(s[1][0], s[1][1]), pack16<TYPE>(s[0][PER - 2], s[0][PER - 1]),
                                    pack16<TYPE>(s[1][PER - 2], s[1][PER - 1])};
#pragma unroll
            for (int t = 0; t < TILES; ++t) {            // column g of product t is channel 64 (t / 8) + 8 g + t % 8
                const int db = t >> 3, x = (t & 7) >> 1;
                const uint32_t pick = t & 1 ? 0x7632u : 0x5410u;
                mma16816<TYPE>(o[t], pf, __byte_perm(w[0][db][x], w[1][db][x], pick), __byte_perm(w[2][db][x], w[3][db][x], pick));
            }
        }
        if (more) load_v(chunk + WARPS);
    }
    // ---- the warps' results, then the thread blocks'
#pragma unroll
    for (int x = 0; x < 2; ++x) {
#pragma unroll
        for (int z = NARROW ? 4 : 1; z < (NARROW ? 32 : 4); z <<= 1) l[x] += __shfl_xor_sync(0xffffffffu, l[x], z);
        const int r = NARROW ? 2 * c + x : g + 8 * x;
        if (NARROW ? g == 0 : c == 0) {
            m_sh[warp][r] = m[x];
            l_sh[warp][r] = l[x];
        }
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            float* const to = o_sh[warp][r];
            if constexpr (NARROW) {
                to[8 * g + t] = o[t][x];
                to[8 * g + (D == 128 ? 64 + t : t + 4)] = o[t][2 + x];
            } else {
                to[64 * (t >> 3) + 8 * (2 * c) + (t & 7)] = o[t][2 * x];
                to[64 * (t >> 3) + 8 * (2 * c + 1) + (t & 7)] = o[t][2 * x + 1];
            }
        }
    }
    __syncthreads();
    if (threadIdx.x < ROWS) {
        const int r = threadIdx.x;
        float top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int x = 0; x < WARPS; ++x) top = fmaxf(top, m_sh[x][r]);
#pragma unroll
        for (int x = 0; x < WARPS; ++x) {
            const float f = m_sh[x][r] == -INFINITY ? 0.f : ptx::ex2(m_sh[x][r] - top);
            weight[x][r] = f;
            sum = fmaf(f, l_sh[x][r], sum);
        }
        m_sh[0][r] = top;
        l_sh[0][r] = sum;
    }
    __syncthreads();
    for (int x = threadIdx.x; x < ROWS * D; x += 32 * WARPS) {
        const int r = x / D, d = x % D;
        float sum = 0.f;
#pragma unroll
        for (int y = 0; y < WARPS; ++y) sum = fmaf(weight[y][r], o_sh[y][r][d], sum);
        o_sh[0][r][d] = sum;
    }
    grid_dependency_launch();
    cluster_sync();
    // this thread block's share of the tile, two channels a thread
    const uint32_t o_at = ptx::smem_u32(&o_sh[0][0][0]), m_at = ptx::smem_u32(&m_sh[0][0]), l_at = ptx::smem_u32(&l_sh[0][0]);
    for (int x = rank * 32 * WARPS + threadIdx.x; x < n_rows * (D / 2); x += size * 32 * WARPS) {
        const int r = x / (D / 2), d = 2 * (x % (D / 2)), head = r / p.w.n_q, i = r - head * p.w.n_q;
        float top = -INFINITY, sum = 0.f, a = 0.f, bb = 0.f;
        for (int y = 0; y < size; ++y) top = fmaxf(top, peer_float(m_at + 4 * r, y));
        for (int y = 0; y < size; ++y) {
            const float my = peer_float(m_at + 4 * r, y), f = my == -INFINITY ? 0.f : ptx::ex2(my - top);
            sum = fmaf(f, peer_float(l_at + 4 * r, y), sum);
            a = fmaf(f, peer_float(o_at + 4 * (r * (D + 4) + d), y), a);
            bb = fmaf(f, peer_float(o_at + 4 * (r * (D + 4) + d + 1), y), bb);
        }
        if (i >= rows) continue;                         // a place behind the sequence's rows
        const float inv = sum > 0.f ? 1.f / sum : 0.f;   // a row that sees nothing: zeros
        *reinterpret_cast<uint32_t*>(p.out.row(b, hk * p.group + head, i) + 2 * d) = pack16<TYPE>(a * inv, bb * inv);
        if (p.lse && d == 0)
            p.lse[((long long)b * p.H + hk * p.group + head) * p.w.n_q + i] = sum > 0.f ? (top + log2f(sum)) * 0.69314718055994531f : -INFINITY;
    }
    cluster_sync();                                      // no thread block leaves while others read its shared memory
}

}  // namespace

bool window_rows_fit(const rapid3_window* w) { return (long long)(w->H / w->H_kv) * w->n_q <= MAX_ROWS; }

cudaError_t launch_window_rows(const rapid3_window* w, const rapid3_rows* q, const rapid3_rows* k, const rapid3_rows* v, const rapid3_rows* out,
                               float* lse, cudaStream_t s) {
    RowsParams p;
    p.w = rule_of(w);
    p.q = rows_arg(q);
    p.k = rows_arg(k);
    p.v = rows_arg(v);
    p.out = rows_arg(out);
    p.lse = lse;
    p.H = w->H;
    p.H_kv = w->H_kv;
    p.group = w->H / w->H_kv;
    p.scale_log2 = w->softmax_scale * 1.4426950408889634f;
    const bool bf = w->type == RAPID3_BF16;
    const auto pick = [&](auto wide, auto wide16, auto narrow, auto narrow16) { return p.group * w->n_q > 8 ? (bf ? wide : wide16) : (bf ? narrow : narrow16); };
    const auto kernel = w->D == 128 ? pick(window_rows_kernel<RAPID3_BF16, 128, false>, window_rows_kernel<RAPID3_F16, 128, false>,
                                           window_rows_kernel<RAPID3_BF16, 128, true>, window_rows_kernel<RAPID3_F16, 128, true>)
                                    : pick(window_rows_kernel<RAPID3_BF16, 64, false>, window_rows_kernel<RAPID3_F16, 64, false>,
                                           window_rows_kernel<RAPID3_BF16, 64, true>, window_rows_kernel<RAPID3_F16, 64, true>);
    // Keys that a sequence's rows may see, and how many thread blocks share them: of the cluster sizes that leave every warp a chunk the one
    // with the least estimated time -- waves of thread blocks, each 4 us and its keys at D / 4 bytes a ns (what its loads on their way allow), or at its share of the SM's 44.
    // Measured, us, sizes 1, 2, 4, 8: 512 pairs of 4100 keys at D = 128 229, 196, 187, 234; 128 pairs of 9000 at D = 64 size 4 56, 8 60, 16 86.  Sixteen
    // need an opt-in and a whole group of SMs, and are left to launches that they alone spread over more SMs.
    long long keys = w->n_kv;
    if (w->left >= 0 && w->n_full == 0) keys = std::min<long long>(keys, (long long)w->left + 1 + w->n_q + w->n_sink);
    const long long pairs = (long long)w->B * w->H_kv;
    const int resident = p.group * w->n_q > 8 ? 2 : w->D == 128 ? 3 : 4;
    int size = 1;
    double least = 0.0;
    for (int x = 1; x <= MAX_CLUSTER; x *= 2) {
        if (x > 1 && (keys < (long long)CHUNK * WARPS * x || (x > 8 && pairs * x > SM_COUNT))) break;
        const long long blocks = pairs * x, per_sm = std::min<long long>(resident, (blocks + SM_COUNT - 1) / SM_COUNT);
        const long long waves = (blocks + resident * SM_COUNT - 1) / (resident * SM_COUNT);
        const double ns = waves * (4000.0 + (double)keys / x * 4 * w->D / std::min(w->D / 4.0, 44.0 / per_sm));
        if (x == 1 || ns < least) {
            least = ns;
            size = x;
        }
    }
    if (size > 8) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return e;
    }
    return launch_kernel_cluster(kernel, dim3((unsigned)(pairs * size)), dim3(32 * WARPS), 0, s, size, p);
}
